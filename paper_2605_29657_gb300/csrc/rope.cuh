// rope.cuh -- turning rows by their positions: what occam_rope and the append that turns
// keys on their way share (internal header).
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace occam {

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

// Cosine and sine of x f (a position and a frequency), formed in two terms (see rope.cu).
__device__ __forceinline__ void rope_angle(float x, float f, float& c, float& s) {
  const float hi = x * f, lo = fmaf(x, f, -hi);
  const float k = rintf(hi * 0.15915494f);
  const float r = fmaf(-k, 6.2831855f, hi);           // exact
  const float rest = fmaf(-k, -1.7484555e-7f, lo);    // 2 pi - 6.2831855f
  const float a = r + rest, e = (r - a) + rest;       // the angle as a + e
  float sh, ch;
  sincosf(a, &sh, &ch);
  c = fmaf(-sh, e, ch);
  s = fmaf(ch, e, sh);
}

// Thread `at` of (row, unit of 2V values), head group `group` of both tensors. AHEAD heads' loads are in flight together
// (by default: two of 16-bit values cost occam_rope more registers than they gain).
template <typename E, int V, bool ADJ, int AHEAD = sizeof(E) == 4 ? 2 : 1>
__device__ __forceinline__ void rope_rows(const RopeParams& p, int64_t at, int group) {
  using VecT = Vec<E, V>;
  const int units = p.dim / (2 * V), turn = p.half / V;
  const int64_t row = at / units;
  const int u = (int)(at - row * units);
  if (row >= p.rows) return;
  const bool first = group < p.groups0;
  const occam_rope_tensor& t = first ? p.t[0] : p.t[1];
  const int h0 = (group - (first ? 0 : p.groups0)) * p.hpt;
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
      rope_angle((float)p.pos[ax * p.pos_stride + row], p.freq[pair], c[i], s[i]);
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
  for (int h = h0; h < h1; h += AHEAD) {
    VecT v0[AHEAD], v1[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (h + k < h1) {
        const E* from = src + (h + k) * t.src_head;
        v0[k] = *reinterpret_cast<const VecT*>(from + d0);
        v1[k] = *reinterpret_cast<const VecT*>(from + d1);
      }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (h + k < h1) {
        E* to = dst + (h + k) * t.dst_head;
        turn_pair(v0[k], v1[k]);
        *reinterpret_cast<VecT*>(to + d0) = v0[k];
        *reinterpret_cast<VecT*>(to + d1) = v1[k];
      }
  }
}

}  // namespace occam
