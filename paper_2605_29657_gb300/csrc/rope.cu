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
#include <algorithm>

#include "common.cuh"
#include "cache.cuh"
#include "nvtx.cuh"
#include "overlap.cuh"
#include "rope.cuh"

using namespace occam;

namespace {

// grid: x over (row, unit of 2V values), y over head groups of both tensors
template <typename E, int V, bool ADJ>
__global__ void __launch_bounds__(256) rope_kernel(RopeParams p) {
  pdl_wait();
  rope_rows<E, V, ADJ>(p, (int64_t)blockIdx.x * blockDim.x + threadIdx.x, blockIdx.y);
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
