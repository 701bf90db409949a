// append_rope.cu -- occam_cache_append_rope: keys turned by their positions on
// the way into the paged 8-bit cache, values beside them, and the queries turned by a second launch
// that overlaps with the first.
//
// A CTA takes one touched page and some heads of K or of V. Cosines and sines of the page's
// tokens are computed once, into shared memory, and serve all its heads of K; the turned values stay
// in registers as fp32 between the block's maximum and the rounding, so keys are rounded once, to their
// codes. The queries are turned by a launch of their own (rope_rows) that starts while this one ends. Bound by HBM:
// queries 2 bytes read and written, keys and values 2 read and 1 written a value: 20 k rows of 32 + 32 + 32 heads of 128 in
// 178 us, 0.70 of a plain copy (keys and values 117 us of it: partly filled pages, and a maximum before the first store).
// A single row a sequence: 13 us, a chain of offsets, table, row, scale.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "append.cuh"
#include "nvtx.cuh"
#include "overlap.cuh"
#include "rope.cuh"
#include "tc5.cuh"

using namespace occam;

namespace {

constexpr int kThreads = 256;

struct EnterParams {
  AppendParams a;
  RopeParams q;          // rows and angles; the queries are t[0]
  int k_heads, v_heads;  // heads a CTA takes of K, of V
  int k_parts, parts;    // CTAs a page for K; in all
};

template <int V>
struct Raw;
template <>
struct Raw<8> {
  uint4 w;
  static constexpr int kWords = 4;
};
template <>
struct Raw<4> {
  uint2 w;
  static constexpr int kWords = 2;
};
template <>
struct Raw<1> {
  uint16_t w;
  static constexpr int kWords = 1;
};
template <bool BF16, int V>
__device__ __forceinline__ void unpack(const Raw<V>& r, float* x) {
  if constexpr (V == 1) {
    x[0] = BF16 ? __uint_as_float((uint32_t)r.w << 16) : __half2float(__ushort_as_half(r.w));
  } else {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&r.w);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      const float2 f = BF16 ? make_float2(bf16_lo(w[i]), bf16_hi(w[i])) : __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}
__device__ __forceinline__ float2 at2(const float* x) { return make_float2(x[0], x[1]); }
// V values to codes at `to`
template <int V>
__device__ __forceinline__ void put_codes(uint8_t* to, const float* x) {
  if constexpr (V == 8) {
    const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
    *reinterpret_cast<uint2*>(to) = make_uint2(f32_codes4(lo), f32_codes4(hi));
  } else if constexpr (V == 4) {
    const float lo[4] = {x[0], x[1], x[2], x[3]};
    *reinterpret_cast<uint32_t*>(to) = f32_codes4(lo);
  } else {
    *to = (uint8_t)f32x2_e4m3x2(x[0], 0.f);
  }
}
// (a scale that is no power of two comes only with a cache whose scales the caller made: kept out of the way of the others)
__device__ __noinline__ float divide(float x, float s) { return x / s; }

// Bytes of a head's rows on their way, each thread its own
template <int V, int NU>
constexpr int kRingBytes = V > 1 ? NU * 2 * kThreads * V * 2 : 0;
template <int V>
__device__ __forceinline__ void copy_async(Raw<V>* to, const uint16_t* from) {
  if constexpr (V == 8)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(to)), "l"(from), "n"(V * 2) : "memory");
}

// V: values of a vector; a unit is two vectors (of pairs, or side by side where nothing is turned). NU: units a
// thread holds of a block at most.
template <bool BF16, int D, int V, bool ADJ, int NU>
__global__ void __launch_bounds__(kThreads, NU * V <= 16 ? 4 : 2) enter_kernel(EnterParams e) {
  extern __shared__ __align__(16) unsigned char smem[];
  Raw<V>* ring = reinterpret_cast<Raw<V>*>(smem) + threadIdx.x;  // [unit][its two vectors][thread]
  // Cosines and sines of each token: (c, s) a pair; where pairs are turned by twos (c, c, s, s), those that a row's
  // threads read together next to one another.
  float* turn = reinterpret_cast<float*>(smem + kRingBytes<V, NU>);
  constexpr bool TWO = V > 1 && !ADJ;
  __shared__ float sh_max[2][kThreads / 32];
  pdl_wait();
  pdl_trigger();  // the queries' launch may begin
  const AppendParams& p = e.a;
  const int64_t w = (int64_t)blockIdx.x / e.parts;
  // (by turns: blocks go to SMs round robin, and an SM that always got the parts of K would be last)
  const int part = (int)((blockIdx.x + w) % e.parts);
  const bool is_k = part < e.k_parts;
  if ((int)blockIdx.x == e.parts) record_backward(p);  // (the second slot: an early CTA, and idle where every sequence has a token)
  const int refused = p.c.status[1] & kRefused;  // (no CTA of this launch sets it)
  const int T = p.c.T, H = p.c.heads;
  // The slot's sequence. Up to 255 of them are looked at at once, with their lengths: two rounds of loads instead of six.
  __shared__ struct {
    int64_t r0, r1;
    int i, seq, len;
  } at;
  if (p.n < kThreads) {
    const int t = threadIdx.x;
    const int64_t r = t <= p.n ? p.row_off[t] : 0;
    const int mine = t < p.n ? p.seqs[t] : -1;
    const int held = (unsigned)mine < (unsigned)p.c.max_seqs ? p.c.length[mine] : -1;
    const int before = __syncthreads_count(t <= p.n && (r >> p.c.log2T) + 2 * (int64_t)t <= w);  // those that begin at or before it
    const int found = min(max(before - 1, 0), p.n - 1);
    if (t == found) {
      at.r0 = r;
      at.i = found;
      at.seq = mine;
      at.len = held;
    }
    if (t == found + 1) at.r1 = r;
  } else if (threadIdx.x < 32) {
    const int found = slot_sequence(p.row_off, p.n, p.c.log2T, w);
    if (threadIdx.x == 0) {
      at.r0 = p.row_off[found];
      at.r1 = p.row_off[found + 1];
      at.i = found;
      at.seq = p.seqs[found];
      at.len = (unsigned)at.seq < (unsigned)p.c.max_seqs ? p.c.length[at.seq] : -1;
    }
  }
  __syncthreads();
  const int i = at.i, seq = at.seq, len = at.len;
  const int64_t r0 = at.r0, r1 = at.r1, local = w - ((r0 >> p.c.log2T) + 2 * (int64_t)i);
  if (refused) return;
  if (local < 0 && r0 <= p.total_rows) return;  // rows before row_off[0] belong to no sequence
  if (!(r0 >= 0 && r1 >= r0 && r1 <= p.total_rows && len >= r1 - r0 && len <= (int64_t)p.c.max_pages * T)) {
    if (threadIdx.x == 0) set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
    return;
  }
  const int start = len - (int)(r1 - r0);  // position of row r0
  if (local > (len >> p.c.log2T)) return;  // (a slot past the rows)
  const int slot = (start >> p.c.log2T) + (int)local;
  if (slot >= p.c.max_pages) return;
  const int t0 = max(start - slot * T, 0), t1 = min(len - slot * T, T);  // new tokens of this page
  if (t1 <= t0) return;
  const int64_t row0 = r0 + (int64_t)slot * T - start + t0;
  if (!in_bounds(i >= 0 && i < p.n && row0 >= r0 && row0 + t1 - t0 <= r1, p.c.status, kSiteAppendRow)) return;
  const int64_t ld = is_k ? p.k_row : p.v_row;
  const uint16_t* src = static_cast<const uint16_t*>(is_k ? p.k : p.v) + row0 * ld;
  const int h0 = is_k ? part * e.k_heads : (part - e.k_parts) * e.v_heads;
  const int h1 = min(h0 + (is_k ? e.k_heads : e.v_heads), H);

  constexpr int UPR = D / (2 * V), STEP = kThreads / UPR;  // units of a row; rows between a thread's units
  const int half = e.q.half, rows = t1 - t0;
  // this thread's units: rows tok0, tok0 + STEP, ..; places of the two vectors; the first pair (-1: not turned)
  const int u = threadIdx.x % UPR, tok0 = threadIdx.x / UPR;
  const int pair = is_k && u < half / V ? u * V : -1;
  const int d0 = pair >= 0 && !ADJ ? V * u : 2 * V * u, d1 = pair >= 0 && !ADJ ? d0 + half : d0 + V;
  // A head's rows come by asynchronous copies, the next head's while one is in hand (single values of 2 bytes by loads).
  auto held = [&](int n, int which) { return ring + (n * 2 + which) * kThreads; };
  auto fetch = [&](int h) {
    if constexpr (V > 1) {
      if (h < h1) {
        const uint16_t* from = src + tok0 * ld + h * D;
#pragma unroll
        for (int n = 0; n < NU; ++n)
          if (tok0 + n * STEP < rows) {
            copy_async<V>(held(n, 0), from + n * STEP * ld + d0);
            copy_async<V>(held(n, 1), from + n * STEP * ld + d1);
          }
      }
      cp_async_commit();
    }
  };
  fetch(h0);
  const int page = p.c.table[(int64_t)seq * p.c.max_pages + slot];
  if ((unsigned)page >= (unsigned)p.c.pages || p.c.refs[page] != 1) {  // no page, or one that other sequences hold
    if (threadIdx.x == 0) set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
    return;
  }
  const int64_t block = ((int64_t)p.layer * p.c.pages + page) * H;
  if (is_k) {
    for (int x = threadIdx.x; x < rows * half; x += kThreads) {
      const int tok = x / half, i = x - tok * half;
      int ax = e.q.axis[i];
      ax = (unsigned)ax < (unsigned)e.q.axes ? ax : 0;
      float* to = turn + 2 * x;
      if (TWO) to = turn + 2 * tok * half + 4 * (i % V / 2 * (half / V) + i / V) + (i & 1);
      rope_angle((float)e.q.pos[ax * e.q.pos_stride + row0 + tok], e.q.freq[i], to[0], to[TWO ? 2 : 1]);
    }
    __syncthreads();
  }
  for (int h = h0; h < h1; ++h) {
    float x[NU][2 * V];
    float amax = 0.f;
    if constexpr (V > 1) cp_async_wait<0>();
#pragma unroll
    for (int n = 0; n < NU; ++n) {
      if (tok0 + n * STEP >= rows) continue;
      if constexpr (V > 1) {
        unpack<BF16, V>(*held(n, 0), x[n]);
        unpack<BF16, V>(*held(n, 1), x[n] + V);
      } else {
        const uint16_t* from = src + (tok0 + n * STEP) * ld + h * D;
        unpack<BF16, V>(Raw<V>{from[d0]}, x[n]);
        unpack<BF16, V>(Raw<V>{from[d1]}, x[n] + V);
      }
      if (pair >= 0) {
        const float* cs = turn + 2 * (tok0 + n * STEP) * half + (TWO ? 4 * u : 2 * pair);
        if constexpr (TWO) {
#pragma unroll
          for (int k = 0; k < V; k += 2) {
            const float4 t = *reinterpret_cast<const float4*>(cs + 2 * k * (half / V));
            const float2 c = make_float2(t.x, t.y), sn = make_float2(t.z, t.w), y = at2(x[n] + k), z = at2(x[n] + V + k);
            // (rounded as below and in rope_rows: every vector width, which the queries' alignment chooses too, gives the same codes)
            const float2 e0 = tc::fma2(y, c, tc::mul2(z, make_float2(-sn.x, -sn.y))), e1 = tc::fma2(z, c, tc::mul2(y, sn));
            x[n][k] = e0.x;
            x[n][k + 1] = e0.y;
            x[n][V + k] = e1.x;
            x[n][V + k + 1] = e1.y;
          }
        } else {
#pragma unroll
          for (int k = 0; k < V; ++k) {
            float& e0 = x[n][ADJ ? 2 * k : k];
            float& e1 = x[n][ADJ ? 2 * k + 1 : V + k];
            const float c = cs[2 * k], sn = cs[2 * k + 1], y = e0, z = e1;
            e0 = fmaf(y, c, -__fmul_rn(z, sn));
            e1 = fmaf(z, c, __fmul_rn(y, sn));
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 2 * V; k += 2) amax = tc::fmax3(amax, fabsf(x[n][k]), fabsf(x[n][k + 1]));  // (passes over NaN)
    }
    fetch(h + 1);  // (in the place of what this thread has just read)
    if (amax == INFINITY) {  // the largest finite value counts
      amax = 0.f;
#pragma unroll
      for (int n = 0; n < NU; ++n)
        if (tok0 + n * STEP < rows)
#pragma unroll
          for (int k = 0; k < 2 * V; ++k) amax = fmaxf(amax, finite_abs(x[n][k]));
    }
    amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax)));
    float* r = sh_max[h & 1];
    if ((threadIdx.x & 31) == 0) r[threadIdx.x >> 5] = amax;
    uint8_t* codes = (is_k ? p.c.k : p.c.v) + (block + h) * T * D;
    float* scale = (is_k ? p.c.k_scale : p.c.v_scale) + block + h;
    const float was = t0 > 0 ? *scale : 0.f;
    __syncthreads();  // (and every thread has `was`)
#pragma unroll
    for (int k = 0; k < kThreads / 32; ++k) amax = fmaxf(amax, r[k]);
    const float need = block_scale(amax);
    const float now = was > need ? was : need;  // older tokens keep at least their scale
    if (t0 > 0 && now > was) {
      // the held codes, rounded again to the larger scale
      const float ratio = was / now;
      for (int y = threadIdx.x; y < t0 * D / 16; y += kThreads) {
        uint4 c = reinterpret_cast<uint4*>(codes)[y];
        uint32_t* cw = reinterpret_cast<uint32_t*>(&c);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float f[4];
          codes4_f32(cw[j], f);
#pragma unroll
          for (int m = 0; m < 4; ++m) f[m] *= ratio;
          cw[j] = f32_codes4(f);
        }
        reinterpret_cast<uint4*>(codes)[y] = c;
      }
    }
    const bool exact = is_pow2(now);
    const float inv = 1.f / now;
    uint8_t* to = codes + (t0 + tok0) * D;
#pragma unroll
    for (int n = 0; n < NU; ++n) {
      if (tok0 + n * STEP >= rows) continue;
      if (exact) {
#pragma unroll
        for (int k = 0; k < 2 * V; k += 2) {
          const float2 y = tc::mul2(at2(x[n] + k), make_float2(inv, inv));
          x[n][k] = y.x;
          x[n][k + 1] = y.y;
        }
      } else {
#pragma unroll
        for (int k = 0; k < 2 * V; ++k) x[n][k] = divide(x[n][k], now);
      }
      put_codes<V>(to + n * STEP * D + d0, x[n]);
      put_codes<V>(to + n * STEP * D + d1, x[n] + V);
    }
    if (threadIdx.x == 0) *scale = now;
  }
}

template <bool BF16, int D, int V, bool ADJ, int NU>
int launch_units(const EnterParams& e, int64_t grid, cudaStream_t st) {
  const int64_t tokens = std::min<int64_t>(e.a.c.T, e.a.total_rows);
  const size_t smem = kRingBytes<V, NU> + (size_t)tokens * e.q.half * sizeof(float2);
  static std::atomic<uint64_t> ready{0};  // devices whose shared memory limit is raised
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return OCCAM_ERR_CUDA;
  if (!((ready.load(std::memory_order_acquire) >> dev) & 1)) {
    if (cudaFuncSetAttribute(enter_kernel<BF16, D, V, ADJ, NU>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             kRingBytes<V, NU> + 128 * (D / 2) * 8) != cudaSuccess)
      return OCCAM_ERR_CUDA;
    ready.fetch_or(uint64_t(1) << dev, std::memory_order_release);
  }
  return launch_after(enter_kernel<BF16, D, V, ADJ, NU>, dim3((unsigned)grid), kThreads, smem, st, e) ? OCCAM_OK : OCCAM_ERR_CUDA;
}

// The queries. Behind a launch for K and V (BEHIND) they need nothing of it but that it is done when they are: what came
// before it was complete when it let this launch begin.
template <bool BF16, int V, bool ADJ, bool BEHIND>
__global__ void __launch_bounds__(kThreads) queries_kernel(RopeParams p) {
  using E = typename std::conditional<BF16, __nv_bfloat16, __half>::type;
  if (!BEHIND) pdl_wait();
  rope_rows<E, V, ADJ>(p, (int64_t)blockIdx.x * kThreads + threadIdx.x, blockIdx.y);
  if (BEHIND) pdl_wait();
}

template <bool BF16, int D, int V, bool ADJ>
int launch_pairing(const EnterParams& e, int64_t grid, dim3 q_grid, cudaStream_t st) {
  if (grid > 0x7fffffff) return OCCAM_ERR_UNSUPPORTED;
  if (grid > 0) {
    // units of a block a thread: page_tokens * D / (2 V) / 256
    constexpr int U64 = std::max(64 * D / (2 * V * kThreads), 1);
    const int rc = e.a.c.T <= 64 ? launch_units<BF16, D, V, ADJ, U64>(e, grid, st) : launch_units<BF16, D, V, ADJ, 2 * U64>(e, grid, st);
    if (rc != OCCAM_OK) return rc;
  }
  const bool ok = e.q.t[0].heads == 0 || (grid > 0 ? launch_after(queries_kernel<BF16, V, ADJ, true>, q_grid, kThreads, 0, st, e.q)
                                                   : launch_after(queries_kernel<BF16, V, ADJ, false>, q_grid, kThreads, 0, st, e.q));
  return ok && cudaGetLastError() == cudaSuccess ? OCCAM_OK : OCCAM_ERR_CUDA;
}

template <bool BF16, int D>
int launch_dim(const EnterParams& e, int v, bool adj, int64_t grid, dim3 q, cudaStream_t st) {
  if (v == 8) return adj ? launch_pairing<BF16, D, 8, true>(e, grid, q, st) : launch_pairing<BF16, D, 8, false>(e, grid, q, st);
  if (v == 4) return adj ? launch_pairing<BF16, D, 4, true>(e, grid, q, st) : launch_pairing<BF16, D, 4, false>(e, grid, q, st);
  return adj ? launch_pairing<BF16, D, 1, true>(e, grid, q, st) : launch_pairing<BF16, D, 1, false>(e, grid, q, st);
}

}  // namespace

#define OCCAM_TRY(x)                 \
  do {                               \
    int _rc = (x);                   \
    if (_rc != OCCAM_OK) return _rc; \
  } while (0)

extern "C" int occam_cache_append_rope(const occam_cache* cache, const occam_append_rope_args* a, void* workspace,
                                       size_t workspace_bytes, occam_stream_t stream) {
  const NvtxRange nvtx("occam_cache_append_rope");
  launch_counter() = 0;
  OCCAM_TRY(check_cache(cache));
  if (!a) return OCCAM_ERR_INVALID_ARG;
  if (a->dtype != OCCAM_BF16 && a->dtype != OCCAM_F16) return OCCAM_ERR_UNSUPPORTED;
  const int dim = cache->dim;
  if (a->layer < 0 || a->layer >= cache->layers || a->total_rows < 0 || a->total_rows > 0x7fffffff || a->n < 0 ||
      a->n > cache->max_seqs || a->rot < 2 || a->rot > dim || (a->rot & 1) || a->axes < 1 || a->axes > 8 || a->pos_stride < 0 ||
      (a->pairing != OCCAM_ROPE_HALF && a->pairing != OCCAM_ROPE_ADJACENT))
    return OCCAM_ERR_INVALID_ARG;
  CacheWs w;
  OCCAM_TRY(check_cache_ws(cache, 0, workspace, workspace_bytes, &w));
  if (a->total_rows == 0) return OCCAM_OK;
  if (!a->positions || !a->inv_freq || !a->axis) return OCCAM_ERR_INVALID_ARG;
  const int64_t row = (int64_t)cache->heads * dim;
  if (a->n > 0 && (!a->k || !a->v || !a->seqs || !a->row_off || !aligned16(a->k) || !aligned16(a->v) || a->k_row < row ||
                   a->v_row < row || (a->k_row & 7) || (a->v_row & 7)))
    return OCCAM_ERR_INVALID_ARG;
  EnterParams e{};
  uintptr_t bits = 0;  // of the queries' addresses and strides
  if (a->q) {
    const occam_rope_tensor& t = *a->q;
    if (!t.src || !t.dst || t.heads < 1 || t.heads > 65535 || t.src_row < 0 || t.src_head < 0 || t.dst_row < 0 || t.dst_head < 0)
      return OCCAM_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(t.src) | reinterpret_cast<uintptr_t>(t.dst)) & 1) return OCCAM_ERR_INVALID_ARG;
    if ((a->total_rows > 1 && t.dst_row < dim) || (t.heads > 1 && t.dst_head < dim)) return OCCAM_ERR_INVALID_ARG;
    if (t.src == t.dst && (t.src_row != t.dst_row || t.src_head != t.dst_head)) return OCCAM_ERR_INVALID_ARG;
    // no value is written that another thread may still read, or writes too
    const Extent to = extent(t.dst, a->total_rows, t.dst_row, t.heads, t.dst_head, dim, 2);
    if (meets_itself(to) || (t.src != t.dst && meet(to, extent(t.src, a->total_rows, t.src_row, t.heads, t.src_head, dim, 2))))
      return OCCAM_ERR_INVALID_ARG;
    if (a->n > 0 && (meet(to, extent(a->k, a->total_rows, a->k_row, cache->heads, dim, dim, 2)) ||
                     meet(to, extent(a->v, a->total_rows, a->v_row, cache->heads, dim, dim, 2))))
      return OCCAM_ERR_INVALID_ARG;
    bits = reinterpret_cast<uintptr_t>(t.src) | reinterpret_cast<uintptr_t>(t.dst) |
           (uintptr_t)((t.src_row | t.src_head | t.dst_row | t.dst_head) * 2);
    e.q.t[0] = t;
  }
  if (a->n == 0 && !a->q) return OCCAM_OK;
  e.a.c = cache_dev(cache, workspace, w);
  e.a.layer = a->layer;
  e.a.n = a->n;
  e.a.total_rows = a->total_rows;
  e.a.k_row = a->k_row;
  e.a.v_row = a->v_row;
  e.a.k = a->k;
  e.a.v = a->v;
  e.a.seqs = a->seqs;
  e.a.row_off = a->row_off;
  e.q.rows = a->total_rows;
  e.q.dim = dim;
  e.q.half = a->rot / 2;
  e.q.axes = a->axes;
  e.q.pos = a->positions;
  e.q.pos_stride = a->pos_stride;
  e.q.freq = a->inv_freq;
  e.q.axis = a->axis;
  // the widest vector that divides the turned and the copied part and that every address is a multiple of
  int v = 8;
  while (v > 1 && (e.q.half % v || (dim - a->rot) % (2 * v) || (bits & (2 * v - 1)))) v = v == 8 ? 4 : 1;
  // Heads a CTA: as many as leave four CTAs an SM (K: up to 16 share a page's cosines and sines).
  const int64_t sms = cache_sms();
  const int64_t slots = a->n > 0 ? (a->total_rows >> e.a.c.log2T) + 2 * (int64_t)a->n : 0;
  auto share = [&](int64_t ctas, int heads, int most) {
    return (int)std::max<int64_t>(1, std::min<int64_t>({ctas * heads / (sms * 4), (int64_t)heads, (int64_t)most}));
  };
  e.k_heads = share(slots, cache->heads, 16);
  e.v_heads = share(slots, cache->heads, 16);
  e.k_parts = (cache->heads + e.k_heads - 1) / e.k_heads;
  e.parts = e.k_parts + (cache->heads + e.v_heads - 1) / e.v_heads;
  // queries: enough threads to fill the GPU first, then as many heads a thread as amortise the sines
  const int64_t q_blocks = (a->total_rows * (dim / (2 * v)) + kThreads - 1) / kThreads;
  const int q_heads = std::max(e.q.t[0].heads, 1);
  if (q_blocks > 0x7fffffff) return OCCAM_ERR_UNSUPPORTED;
  e.q.hpt = (int)std::max<int64_t>(std::min<int64_t>({q_blocks * q_heads / (sms * 8), (int64_t)q_heads, (int64_t)kMostHeads}), 1);
  e.q.groups0 = (q_heads + e.q.hpt - 1) / e.q.hpt;
  if (e.q.groups0 > 65535) return OCCAM_ERR_UNSUPPORTED;
  const dim3 q_grid((unsigned)q_blocks, (unsigned)e.q.groups0);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const bool adj = a->pairing == OCCAM_ROPE_ADJACENT, bf16 = a->dtype == OCCAM_BF16;
  if (dim == 128) return bf16 ? launch_dim<true, 128>(e, v, adj, slots * e.parts, q_grid, st) : launch_dim<false, 128>(e, v, adj, slots * e.parts, q_grid, st);
  return bf16 ? launch_dim<true, 64>(e, v, adj, slots * e.parts, q_grid, st) : launch_dim<false, 64>(e, v, adj, slots * e.parts, q_grid, st);
}
