// rope.cu -- rotary positions with several axes (occam_rope).
//
// Per row and pair one angle, shared by every head of the queries and keys:
// a thread computes the sines and cosines of its V pairs once and turns those
// pairs of up to `hpt` heads, so the trigonometry is paid once for that many
// vectors. The angle p * f is formed as the rounded product and its rounding error
// (one fused multiply-add) and brought into one turn in two steps (2 pi as a sum of two
// fp32 numbers; the first step is exact), so the result does not lose digits
// at large positions (integers up to 2^24 are exact in fp32). Bound by HBM:
// every value is read and written once. 65,792 rows of 64 heads of 128 dims, bf16:
// 345 us, 6.3 TB/s (0.92 of a plain copy's); 34,813 rows of 32 heads of 72 dims, fp32: 101 us,
// 6.3 TB/s; 64 rows of 40 heads: 5.5 us, the chain of loads, sines and stores.
#include <cuda_fp16.h>

#include <algorithm>

#include "common.cuh"
#include "cache.cuh"
#include "nvtx.cuh"

using namespace occam;

namespace {

struct RopeParams {
  int64_t rows;
  int dim, half, axes, inverse;
  const int32_t* pos;
  int64_t pos_stride;
  const float* freq;
  const int32_t* axis;
  int hpt;          // heads per thread
  int groups0;      // head groups of tensor 0
  occam_rope_tensor t[2];
};

template <typename E>
__device__ __forceinline__ float to_f(E x);
template <>
__device__ __forceinline__ float to_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f<__half>(__half x) { return __half2float(x); }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename E>
__device__ __forceinline__ E from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

constexpr int kMostHeads = 32;  // heads a thread takes at most

template <typename E, int V>
struct alignas(sizeof(E) * V) Vec {
  E x[V];
};

// grid: x over (row, unit of 2V values), y over head groups of both tensors
template <typename E, int V, bool ADJ>
__global__ void __launch_bounds__(256) rope_kernel(RopeParams p) {
  using VecT = Vec<E, V>;
  pdl_wait();
  const int units = p.dim / (2 * V), turn = p.half / V;
  const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t row = at / units;
  const int u = (int)(at - row * units);
  if (row >= p.rows) return;
  const bool first = (int)blockIdx.y < p.groups0;
  const occam_rope_tensor& t = first ? p.t[0] : p.t[1];
  const int h0 = ((int)blockIdx.y - (first ? 0 : p.groups0)) * p.hpt;
  const int h1 = min(h0 + p.hpt, t.heads);
  const bool turned = u < turn;
  // the two vectors of the unit
  const int d0 = turned ? (ADJ ? 2 * V * u : V * u) : 2 * V * u;
  const int d1 = turned && !ADJ ? d0 + p.half : d0 + V;
  float c[V], s[V];
  if (turned) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int pair = u * V + i;
      int ax = p.axis[pair];
      ax = (unsigned)ax < (unsigned)p.axes ? ax : 0;
      const float x = (float)p.pos[ax * p.pos_stride + row], f = p.freq[pair];
      const float hi = x * f, lo = fmaf(x, f, -hi);
      const float k = rintf(hi * 0.15915494f);
      const float r = fmaf(-k, 6.2831855f, hi);           // exact
      const float rest = fmaf(-k, -1.7484555e-7f, lo);    // 2 pi - 6.2831855f
      const float a = r + rest, e = (r - a) + rest;       // the angle as a + e
      float sh, ch;
      sincosf(a, &sh, &ch);
      c[i] = fmaf(-sh, e, ch);
      s[i] = fmaf(ch, e, sh);
      if (p.inverse) s[i] = -s[i];
    }
  }
  const E* src = static_cast<const E*>(t.src) + row * t.src_row;
  E* dst = static_cast<E*>(t.dst) + row * t.dst_row;
  auto turn_pair = [&](VecT& v0, VecT& v1) {
    if (turned) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        E& e0 = ADJ ? (2 * i < V ? v0.x[(2 * i) % V] : v1.x[(2 * i) % V]) : v0.x[i];
        E& e1 = ADJ ? (2 * i + 1 < V ? v0.x[(2 * i + 1) % V] : v1.x[(2 * i + 1) % V]) : v1.x[i];
        const float x = to_f<E>(e0), y = to_f<E>(e1);
        // (the rounding is spelled out, so every vector width gives the same bits)
        e0 = from_f<E>(fmaf(x, c[i], -__fmul_rn(y, s[i])));
        e1 = from_f<E>(fmaf(y, c[i], __fmul_rn(x, s[i])));
      }
    }
  };
  // kAhead heads' loads are in flight together (two of 16-bit values cost more registers than they gain)
  constexpr int kAhead = sizeof(E) == 4 ? 2 : 1;
  for (int h = h0; h < h1; h += kAhead) {
    VecT v0[kAhead], v1[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (h + k < h1) {
        const E* from = src + (h + k) * t.src_head;
        v0[k] = *reinterpret_cast<const VecT*>(from + d0);
        v1[k] = *reinterpret_cast<const VecT*>(from + d1);
      }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (h + k < h1) {
        E* to = dst + (h + k) * t.dst_head;
        turn_pair(v0[k], v1[k]);
        *reinterpret_cast<VecT*>(to + d0) = v0[k];
        *reinterpret_cast<VecT*>(to + d1) = v1[k];
      }
  }
}

template <typename E, int V>
bool launch_v(const RopeParams& p, int adj, dim3 grid, cudaStream_t st) {
  return adj ? launch_after(rope_kernel<E, V, true>, grid, 256, 0, st, p)
             : launch_after(rope_kernel<E, V, false>, grid, 256, 0, st, p);
}

template <typename E>
int launch_t(RopeParams& p, int adj, int n, cudaStream_t st) {
  // the widest vector (16 bytes at most) that divides the turned and the
  // copied part and that every address is a multiple of
  int v = 16 / (int)sizeof(E);
  auto fits = [&](int w) {
    if (p.half % w || (p.dim - 2 * p.half) % (2 * w)) return false;
    const uintptr_t mask = (uintptr_t)w * sizeof(E) - 1;
    for (int i = 0; i < n; ++i) {
      const occam_rope_tensor& t = p.t[i];
      const uintptr_t bits = reinterpret_cast<uintptr_t>(t.src) | reinterpret_cast<uintptr_t>(t.dst) |
                             (uintptr_t)((t.src_row | t.src_head | t.dst_row | t.dst_head) * (int64_t)sizeof(E));
      if (bits & mask) return false;
    }
    return true;
  };
  while (v > 1 && !fits(v)) v >>= 1;
  const int64_t units = p.dim / (2 * v);
  const int64_t blocks = (p.rows * units + 255) / 256;
  if (blocks > 0x7fffffff) return OCCAM_ERR_UNSUPPORTED;
  // Heads per thread: enough threads to fill the GPU first (2048 an SM), then
  // as many heads as amortise the sines (65,792 rows of 64 heads of 128 dims,
  // bf16: 8 heads 377 us, 16 355 us, 32 345 us).
  const int heads = p.t[0].heads + (n > 1 ? p.t[1].heads : 0);
  const int64_t want = (int64_t)cache_sms() * 2048;
  int64_t hpt = blocks * 256 * heads / want;
  p.hpt = (int)(hpt < 1 ? 1 : hpt > kMostHeads ? kMostHeads : hpt);
  p.groups0 = (p.t[0].heads + p.hpt - 1) / p.hpt;
  const int groups = p.groups0 + (n > 1 ? (p.t[1].heads + p.hpt - 1) / p.hpt : 0);
  if (groups > 65535) return OCCAM_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)blocks, (unsigned)groups);
  bool ok = false;
  if (v == 8) {
    if constexpr (sizeof(E) == 2) ok = launch_v<E, 8>(p, adj, grid, st);
  } else if (v == 4) {
    ok = launch_v<E, 4>(p, adj, grid, st);
  } else if (v == 2) {
    ok = launch_v<E, 2>(p, adj, grid, st);
  } else {
    ok = launch_v<E, 1>(p, adj, grid, st);
  }
  return ok && cudaGetLastError() == cudaSuccess ? OCCAM_OK : OCCAM_ERR_CUDA;
}

// A tensor's values as intervals of `width` elements at base + r row + h head.
struct Extent {
  __int128 base, row, head, rows, heads, width;  // base in elements
  __int128 end() const { return base + (rows - 1) * row + (heads - 1) * head + width; }
};
Extent extent(const void* at, int64_t rows, int64_t row, int64_t heads, int64_t head, int64_t dim, int64_t es) {
  Extent e{(__int128)(reinterpret_cast<uintptr_t>(at) / es), row, head, rows, heads, dim};
  if (e.rows == 1 || e.row == 0) e.rows = 1, e.row = 0;      // (a row read again is one row)
  if (e.heads == 1 || e.head == 0) e.heads = 1, e.head = 0;
  if (e.head == e.width) e.width *= e.heads, e.heads = 1, e.head = 0;  // heads side by side are one interval
  return e;
}
// Whether c + n pitch lies in lo .. hi for some n in first .. last (pitch >= 0).
bool reaches(__int128 c, __int128 pitch, __int128 first, __int128 last, __int128 lo, __int128 hi) {
  if (pitch == 0) return lo <= c && c <= hi;
  auto floor_div = [](__int128 a, __int128 b) { return a >= 0 ? a / b : -((-a + b - 1) / b); };
  const __int128 n = std::max(first, -floor_div(c - lo, pitch));  // the least n with c + n pitch >= lo
  return n <= last && c + n * pitch <= hi;
}
// Whether two tensors have an element in common. (Exact, but for tensors that lie within each other with
// rows of different strides, or more than 2^20 pairs of heads with different strides: true.)
bool meet(const Extent& a, const Extent& b) {
  if (a.end() <= b.base || b.end() <= a.base) return false;
  if (a.rows > 1 && b.rows > 1 && a.row != b.row) return true;
  const __int128 pitch = a.rows > 1 ? a.row : b.row, at = a.base - b.base;
  auto rows_meet = [&](__int128 c) { return reaches(c, pitch, 1 - b.rows, a.rows - 1, 1 - a.width, b.width - 1); };
  if (a.heads == 1 || b.heads == 1 || a.head == b.head) {
    const __int128 head = a.heads > 1 ? a.head : b.head;
    for (__int128 h = 1 - b.heads; h < a.heads; ++h)
      if (rows_meet(at + h * head)) return true;
    return false;
  }
  if (a.heads * b.heads > (1 << 20)) return true;
  for (__int128 h = 0; h < a.heads; ++h)
    for (__int128 k = 0; k < b.heads; ++k)
      if (rows_meet(at + h * a.head - k * b.head)) return true;
  return false;
}
// Whether two of a tensor's own (row, head) intervals have an element in common.
bool meets_itself(const Extent& a) {
  if (a.row >= (a.heads - 1) * a.head + a.width || a.rows == 1) return a.heads > 1 && a.head < a.width;
  if (a.heads == 1) return true;  // (rows closer than a row is wide)
  if (a.head >= (a.rows - 1) * a.row + a.width) return a.row < a.width;
  for (__int128 h = 0; h < a.heads; ++h)  // h = 0: rows 1 .. apart
    if (reaches(h * a.head, a.row, h ? 1 - a.rows : 1, a.rows - 1, 1 - a.width, a.width - 1)) return true;
  return false;
}

}  // namespace

extern "C" int occam_rope(int32_t dtype, int64_t rows, int32_t dim, int32_t rot, int32_t pairing, int32_t inverse,
                          const int32_t* positions, int64_t pos_stride, int32_t axes, const float* inv_freq,
                          const int32_t* axis, int32_t n_tensors, const occam_rope_tensor* tensors,
                          occam_stream_t stream) {
  const NvtxRange nvtx("occam_rope");
  launch_counter() = 0;
  if (dtype != OCCAM_BF16 && dtype != OCCAM_F16 && dtype != OCCAM_F32) return OCCAM_ERR_UNSUPPORTED;
  if (dim < 2 || dim > 1024 || (dim & 1)) return OCCAM_ERR_UNSUPPORTED;
  if (rot < 2 || rot > dim || (rot & 1) || rows < 0 || rows > 0x7fffffff || axes < 1 || axes > 8) return OCCAM_ERR_INVALID_ARG;
  if (pairing != OCCAM_ROPE_HALF && pairing != OCCAM_ROPE_ADJACENT) return OCCAM_ERR_INVALID_ARG;
  if (!tensors || n_tensors < 1 || n_tensors > 2 || pos_stride < 0) return OCCAM_ERR_INVALID_ARG;
  if (rows == 0) return OCCAM_OK;
  if (!positions || !inv_freq || !axis) return OCCAM_ERR_INVALID_ARG;
  const uintptr_t es = dtype == OCCAM_F32 ? 4 : 2;
  RopeParams p{};
  Extent to[2], from[2];
  for (int i = 0; i < n_tensors; ++i) {
    const occam_rope_tensor& t = tensors[i];
    if (!t.src || !t.dst || t.heads < 1 || t.heads > 65535 || t.src_row < 0 || t.src_head < 0 || t.dst_row < 0 || t.dst_head < 0)
      return OCCAM_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(t.src) | reinterpret_cast<uintptr_t>(t.dst)) & (es - 1)) return OCCAM_ERR_INVALID_ARG;
    // no value of dst has two places to come from
    if ((rows > 1 && t.dst_row < dim) || (t.heads > 1 && t.dst_head < dim)) return OCCAM_ERR_INVALID_ARG;
    to[i] = extent(t.dst, rows, t.dst_row, t.heads, t.dst_head, dim, es);
    from[i] = extent(t.src, rows, t.src_row, t.heads, t.src_head, dim, es);
    if (meets_itself(to[i])) return OCCAM_ERR_INVALID_ARG;
    // in place means the same strides: a row's values are read before they are written
    if (t.src == t.dst && (t.src_row != t.dst_row || t.src_head != t.dst_head)) return OCCAM_ERR_INVALID_ARG;
    p.t[i] = t;
  }
  // no value is written that another thread may still read, or writes too
  for (int i = 0; i < n_tensors; ++i)
    for (int j = 0; j < n_tensors; ++j) {
      if (i < j && meet(to[i], to[j])) return OCCAM_ERR_INVALID_ARG;
      if (!(i == j && p.t[i].src == p.t[i].dst) && meet(to[i], from[j])) return OCCAM_ERR_INVALID_ARG;
    }
  p.rows = rows;
  p.dim = dim;
  p.half = rot / 2;
  p.axes = axes;
  p.inverse = inverse ? 1 : 0;
  p.pos = positions;
  p.pos_stride = pos_stride;
  p.freq = inv_freq;
  p.axis = axis;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const int adj = pairing == OCCAM_ROPE_ADJACENT;
  if (dtype == OCCAM_F32) return launch_t<float>(p, adj, n_tensors, st);
  if (dtype == OCCAM_F16) return launch_t<__half>(p, adj, n_tensors, st);
  return launch_t<__nv_bfloat16>(p, adj, n_tensors, st);
}
