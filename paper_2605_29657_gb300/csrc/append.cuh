// append.cuh -- what the calls that write rows into the paged cache share (internal header).
#pragma once

#include "cache.cuh"

namespace occam {

struct AppendParams {
  CacheDev c;
  int layer, n;
  int64_t total_rows, k_row, v_row;
  const void* k;
  const void* v;
  const int32_t* seqs;
  const int64_t* row_off;
};

// Offsets that go back are recorded, by one CTA: sequences at such a place take each other's slots, and their pages
// may be looked at by nobody.
__device__ __forceinline__ void record_backward(const AppendParams& p) {
  bool back = false;
  for (int i = threadIdx.x; i < p.n; i += blockDim.x) back |= p.row_off[i + 1] < p.row_off[i];
  if (back) set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
}

// The first index whose slot count passes w: sequence i's pages occupy slots
// [row_off[i] / T + 2 i, row_off[i+1] / T + 2 (i + 1)), at least as many as
// the pages its rows can touch. One warp searches 32 ways at a time.
__device__ __forceinline__ int slot_sequence(const int64_t* row_off, int n, int log2T, int64_t w) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n;  // slot(lo) <= w < slot(hi)
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32;
    const int i = min(lo + (lane + 1) * step, hi);
    const bool past = i >= hi || (row_off[i] >> log2T) + 2 * (int64_t)i > w;
    const unsigned b = __ballot_sync(0xffffffffu, past);
    const int f = __ffs(b) - 1;  // some lane always reaches hi
    const int nh = min(lo + (f + 1) * step, hi);
    lo = lo + f * step;
    hi = nh;
  }
  return lo;
}

template <bool BF16>
__device__ __forceinline__ void unpack8(uint4 r, float (&x)[8]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (BF16) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}

// the largest finite |value| of 8 elements, as a float
template <bool BF16>
__device__ __forceinline__ float amax8(uint4 r) {
  const uint32_t w[4] = {r.x & 0x7fff7fffu, r.y & 0x7fff7fffu, r.z & 0x7fff7fffu, r.w & 0x7fff7fffu};
  // magnitudes order as integers
  uint32_t m = __vmaxu2(__vmaxu2(w[0], w[1]), __vmaxu2(w[2], w[3]));
  m = max(m >> 16, m & 0xffffu);
  if (m >= (BF16 ? 0x7f80u : 0x7c00u)) {  // an infinity or NaN among them
    m = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t a = w[k] >> 16, b = w[k] & 0xffffu, end = BF16 ? 0x7f80u : 0x7c00u;
      m = max(m, max(a < end ? a : 0u, b < end ? b : 0u));
    }
  }
  return BF16 ? __uint_as_float(m << 16) : __half2float(__ushort_as_half((unsigned short)m));
}

// 8 values to codes. (A scale that is no power of two comes only with a cache whose scales the
// caller made: by division, kept out of the way of the others.)
template <bool BF16>
__device__ __forceinline__ uint2 codes8(uint4 r, float inv) {
  float f[8];
  unpack8<BF16>(r, f);
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] *= inv;
  const float lo[4] = {f[0], f[1], f[2], f[3]}, hi[4] = {f[4], f[5], f[6], f[7]};
  return make_uint2(f32_codes4(lo), f32_codes4(hi));
}
template <bool BF16>
__device__ __noinline__ uint2 codes8_by_division(uint4 r, float scale) {
  float f[8];
  unpack8<BF16>(r, f);
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] /= scale;
  const float lo[4] = {f[0], f[1], f[2], f[3]}, hi[4] = {f[4], f[5], f[6], f[7]};
  return make_uint2(f32_codes4(lo), f32_codes4(hi));
}

}  // namespace occam
