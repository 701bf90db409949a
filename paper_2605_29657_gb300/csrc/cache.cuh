// cache.cuh -- shared pieces of the paged 8-bit cache (cache.cu, attend.cu,
// internal header): workspace layout, argument checks, code conversion.
#pragma once

#include <cuda_fp16.h>

#include <utility>

#include "common.cuh"
#include "validate.cuh"

namespace occam {

// Attention workspace: at most kAttendCtas stretches of work leave two partial results of
// up to kAttendRows rows each (the tensor-core kernel: kAttendTcCtas, 256 rows).
constexpr int kAttendCtas = 512;
constexpr int kAttendRows = 16;
constexpr int kAttendTcCtas = 160;
constexpr size_t kAttendPartRows =
    2 * ((size_t)kAttendCtas * kAttendRows > (size_t)kAttendTcCtas * 256 ? (size_t)kAttendCtas * kAttendRows
                                                                         : (size_t)kAttendTcCtas * 256);

inline size_t cache_align(size_t x) { return (x + 255) / 256 * 256; }

// Byte offsets from the workspace base. Everything but status and counters
// is written before it is read within each call.
struct CacheWs {
  size_t status, counters;  // zero between calls (attention's counters: also after a wait that ran out)
  size_t count, lead, head, new_pages, free_list, old_table, list, part_o, part_ml;
  size_t total;
};

inline CacheWs cache_ws(const occam_cache* c, int64_t max_tokens) {
  CacheWs w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = cache_align(off + (bytes ? bytes : 1));
    return o;
  };
  w.status = take(8);
  w.counters = take((size_t)(kAttendCtas + 1) * 4);  // (the last: CTAs that have left)
  w.count = take((size_t)c->max_seqs * 4);
  w.lead = take((size_t)c->max_seqs * 4);
  w.head = take((size_t)(c->max_seqs + 1) * 4);
  w.new_pages = take((size_t)c->max_seqs * 8);
  w.free_list = take((size_t)c->pages * 4);
  w.old_table = take((size_t)c->max_seqs * c->max_pages * 4);
  w.part_o = take(kAttendPartRows * c->dim * 4);
  w.part_ml = take(kAttendPartRows * 8);
  w.list = take((size_t)max_tokens * 4);  // last: its size is the caller's
  w.total = off;
  return w;
}

inline int check_cache(const occam_cache* c) {
  if (!c) return OCCAM_ERR_INVALID_ARG;
  if (c->dim != 64 && c->dim != 128) return OCCAM_ERR_UNSUPPORTED;
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128)
    return OCCAM_ERR_UNSUPPORTED;
  if (c->layers < 1 || c->layers > 65535 || c->pages < 1 || c->pages > (1 << 24) ||
      (int64_t)c->layers * c->pages > 0x7fffffff || c->heads < 1 || c->heads > 1024 || c->max_seqs < 1 ||
      c->max_seqs > 65535 || c->max_pages < 1 || (int64_t)c->max_pages * c->page_tokens >= (int64_t(1) << 31) - 256)
    return OCCAM_ERR_INVALID_ARG;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->table || !c->length || !c->refs) return OCCAM_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v)) return OCCAM_ERR_INVALID_ARG;
  return OCCAM_OK;
}

inline int check_cache_ws(const occam_cache* c, int64_t tokens, void* ws, size_t bytes, CacheWs* w) {
  *w = cache_ws(c, tokens);
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) != 0 || bytes < w->total) return OCCAM_ERR_WORKSPACE;
  return OCCAM_OK;
}

template <typename T>
T* ws_at(void* ws, size_t off) {
  return reinterpret_cast<T*>(static_cast<unsigned char*>(ws) + off);
}

// SMs of the current device
int cache_sms();

// Launches `kern` so that its start overlaps the end of the kernel before it in the stream; the
// kernel itself waits for that one (pdl_wait) before it reads anything.
template <class... P, class... A>
bool launch_after(void (*kern)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  count_launch();
  return cudaLaunchKernelEx(&cfg, kern, std::forward<A>(args)...) == cudaSuccess;
}

// ---------------------------------------------------------------- device
struct CacheDev {
  int layers, pages, heads, T, log2T, max_seqs, max_pages;
  uint8_t* k;
  uint8_t* v;
  float* k_scale;
  float* v_scale;
  int32_t* table;
  int32_t* length;
  int32_t* refs;
  int32_t* status;
};

// Set in the word after the status word by an extend that records an error; both are cleared
// when the status is read. Until then nothing grows and nothing is appended: the rows
// of an append behind it would land on the last tokens that are held.
constexpr int32_t kRefused = 1 << 30;

inline CacheDev cache_dev(const occam_cache* c, void* ws, const CacheWs& w) {
  CacheDev d;
  d.layers = c->layers;
  d.pages = c->pages;
  d.heads = c->heads;
  d.T = c->page_tokens;
  d.log2T = c->page_tokens == 16 ? 4 : c->page_tokens == 32 ? 5 : c->page_tokens == 64 ? 6 : 7;
  d.max_seqs = c->max_seqs;
  d.max_pages = c->max_pages;
  d.k = static_cast<uint8_t*>(c->k);
  d.v = static_cast<uint8_t*>(c->v);
  d.k_scale = c->k_scale;
  d.v_scale = c->v_scale;
  d.table = c->table;
  d.length = c->length;
  d.refs = c->refs;
  d.status = ws_at<int32_t>(ws, w.status);
  return d;
}

// two e4m3 codes (low byte first) as two f16 values, exactly
__device__ __forceinline__ uint32_t e4m3x2_f16x2(uint32_t two) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(two));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x2_f16x2_hi(uint32_t two) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(r) : "r"(two));
  return r;
}
// (lo, hi) to two codes: round to nearest even, saturating; NaN stays NaN
__device__ __forceinline__ uint32_t f32x2_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void codes4_f32(uint32_t w, float (&x)[4]) {
  const uint32_t a = e4m3x2_f16x2(w), b = e4m3x2_f16x2_hi(w);
  const float2 fa = __half22float2(*reinterpret_cast<const __half2*>(&a));
  const float2 fb = __half22float2(*reinterpret_cast<const __half2*>(&b));
  x[0] = fa.x;
  x[1] = fa.y;
  x[2] = fb.x;
  x[3] = fb.y;
}
__device__ __forceinline__ uint32_t f32_codes4(const float (&x)[4]) {
  return f32x2_e4m3x2(x[0], x[1]) | (f32x2_e4m3x2(x[2], x[3]) << 16);
}

// The smallest power of two s, 2^-100 at least, with amax <= 448 s = 1.75 2^8 s
// (amax finite and >= 0): from amax's exponent and mantissa, exactly.
__device__ __forceinline__ float block_scale(float amax) {
  const int b = __float_as_int(amax);
  int e = (b >> 23) - 127 - 8 + ((b & 0x7fffff) > 0x600000 ? 1 : 0);
  e = e < -100 ? -100 : e > 120 ? 120 : e;
  return __int_as_float((e + 127) << 23);
}
// x / s: a product with the exact reciprocal where s is a power of two
// (every scale this library chooses), else a division
__device__ __forceinline__ bool is_pow2(float s) {
  return (__float_as_int(s) & 0x7fffff) == 0 && s >= 1.2e-38f && s <= 8.0e37f;
}
// Adds 1 and returns what was there. What the block wrote before a barrier before this is
// visible to the block whose later arrival sees it. (A fence of every thread
// instead waits for 5 to 25 us while the memory system is busy.)
__device__ __forceinline__ int arrive_count(int32_t* counter) {
  int was;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(was) : "l"(counter) : "memory");
  return was;
}
// |x| if finite, else 0
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a <= 3.4028235e38f ? a : 0.f;
}

}  // namespace occam
