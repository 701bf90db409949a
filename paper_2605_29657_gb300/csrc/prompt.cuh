// prompt.cuh -- what the kernels of a whole prompt's attention (prompt.cu) and
// of its gradient (prompt_grad.cu) share (internal header): parameters, the list
// of items and how CTAs take them, bounded waits.
//
// An item is a block of rows of one sequence and some heads. Items are taken from
// a counter, the first ones by block index: CTAs that had short items take more of them.
// A sequence's heaviest items come first, so that what is left at the end is short.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "cache.cuh"
#include "overlap.cuh"
#include "tc5.cuh"

namespace occam {

struct PromptParams {
  int n, H, Hkv, G, log2P, causal, dim;  // 2^log2P heads of a group are packed as rows of a tile
  int most;                              // items of blocks of rows, of sequences that do not overlap
  int64_t total_rows, total_keys;
  const int64_t* row_off;
  const int64_t* key_off;
  float scale, scale_log2;
  uint16_t* out;
  float* lse;
  int32_t* status;
  int32_t* counters;  // [0] items taken beyond the first of each CTA, [1] CTAs that have left; zero between calls
};

constexpr int64_t kPromptRows = 0x7fffffff - 1023;  // places in a tile behind the last row still fit 32 bits

// The smallest power of two above any factor of a score: never 0, so that a hidden key's -inf stays
constexpr float kLeastFactor = 1.2e-38f;

struct PromptSeq {
  int64_t row0, key0;
  int rows, keys;
};
// Sequence i; no rows and no keys if its offsets do not fit (recorded).
__device__ __forceinline__ PromptSeq prompt_seq(const PromptParams& p, int i) {
  PromptSeq s;
  s.row0 = p.row_off[i];
  const int64_t r1 = p.row_off[i + 1];
  s.key0 = p.key_off[i];
  const int64_t k1 = p.key_off[i + 1];
  if (s.row0 >= 0 && r1 >= s.row0 && r1 <= p.total_rows && s.key0 >= 0 && k1 >= s.key0 && k1 <= p.total_keys) {
    s.rows = (int)(r1 - s.row0);
    s.keys = (int)(k1 - s.key0);
    return s;
  }
  set_status(p.status, OCCAM_ERR_INVALID_ARG);
  s.row0 = s.key0 = 0;
  s.rows = s.keys = 0;
  return s;
}
// Keys that the row at place tok of its sequence sees; none (never fewer) where the rows outnumber the keys.
__device__ __forceinline__ int prompt_limit(const PromptParams& p, int rows, int keys, int tok) {
  return p.causal ? max(keys - rows + tok + 1, 0) : keys;
}

// A CTA's item, told to its roles. Fields after `hb` are the kernel's own.
struct PromptItem {
  int64_t row0, key0;
  int rows, keys;
  int tile, hb;    // the block of rows (or keys) and the block of heads
  int steps;       // 0: there is none, the CTA is done (the gradient's keys: an item without work; nk[1] says that there is none)
  int nk[2];       // steps of each row tile
  int step0, part; // (the gradient's keys) the first step; the part of a divided item, -1: it is whole, -2: there is no such part
};

// How a kernel cuts a sequence: `len` rows (or keys) in blocks of `block`, head blocks inner.
// The prefix sums of item counts over kChunks runs of sequences are in shared memory.
constexpr int kChunks = 128;
struct PromptList {
  long long part[4];
  int first[kChunks + 1];
};

// Block-wide, all threads (at least 128). COUNT(seq) gives a sequence's items; most: what sequences that do not overlap have
// at most. More (offsets that go back and forth over the same rows) is recorded, and there are no items.
template <class Count>
__device__ __forceinline__ void prompt_list(const PromptParams& p, PromptList& l, const Count& count, int most) {
  const int t = threadIdx.x, per = (p.n + kChunks - 1) / kChunks;
  long long mine = 0, incl = 0;
  if (t < kChunks) {
    for (int i = t * per; i < min((t + 1) * per, p.n); ++i) mine += count(prompt_seq(p, i));
    incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, incl, o);
      if ((t & 31) >= o) incl += x;
    }
    if ((t & 31) == 31) l.part[t >> 5] = incl;
  }
  __syncthreads();
  if (t < kChunks) {
    for (int w = 0; w < (t >> 5); ++w) incl += l.part[w];
    const bool over = l.part[0] + l.part[1] + l.part[2] + l.part[3] > most;
    l.first[t + 1] = over ? 0 : (int)incl;
    if (t == 0) {
      l.first[0] = 0;
      if (over) set_status(p.status, OCCAM_ERR_INVALID_ARG);
    }
  }
  __syncthreads();
}
// A CTA's items, taken by one warp: the next one is asked for when one is taken, so that the counter's latency is hidden,
// and the sequence is looked up only where it changes.
struct PromptTaker {
  int next;        // lane 0: the next item (its block's own first)
  int begin, end;  // the present sequence's items
  PromptSeq s;

  __device__ __forceinline__ PromptTaker() : next(blockIdx.x), begin(0), end(0) { s.row0 = s.key0 = s.rows = s.keys = 0; }
  // The item's place among those of sequence s; -1: there is none. COUNT(seq) gives a sequence's items.
  template <class Count>
  __device__ __forceinline__ int take(const PromptParams& p, const PromptList& l, const Count& count) {
    const int lane = threadIdx.x & 31, at = __shfl_sync(0xffffffffu, next, 0);
    if (at >= l.first[kChunks]) return -1;
    if (lane == 0) next = gridDim.x + atomicAdd(&p.counters[0], 1);
    if (at < begin || at >= end) find(p, l, count, at);
    return at - begin;
  }
  template <class Count>
  __device__ __forceinline__ void find(const PromptParams& p, const PromptList& l, const Count& count, int at) {
    const int lane = threadIdx.x & 31, per = (p.n + kChunks - 1) / kChunks;
    int before = 0;
#pragma unroll
    for (int k = 0; k < kChunks / 32; ++k) before += l.first[k * 32 + lane + 1] <= at;
    const int c = __reduce_add_sync(0xffffffffu, before);
    int base = l.first[c];
    for (int i = c * per; i < min((c + 1) * per, p.n); i += 32) {
      PromptSeq x;
      x.row0 = x.key0 = x.rows = x.keys = 0;
      int mine = 0;
      if (i + lane < min((c + 1) * per, p.n)) {
        x = prompt_seq(p, i + lane);
        mine = count(x);
      }
      int incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      const unsigned past = __ballot_sync(0xffffffffu, at < base + incl);
      if (past) {
        const int from = __ffs(past) - 1;
        end = base + __shfl_sync(0xffffffffu, incl, from);
        begin = end - __shfl_sync(0xffffffffu, mine, from);
        s.row0 = __shfl_sync(0xffffffffu, x.row0, from);
        s.key0 = __shfl_sync(0xffffffffu, x.key0, from);
        s.rows = __shfl_sync(0xffffffffu, x.rows, from);
        s.keys = __shfl_sync(0xffffffffu, x.keys, from);
        return;
      }
      base += __shfl_sync(0xffffffffu, incl, 31);
    }
  }
};

// The last CTA to leave clears the counters, whatever happened: the next call has to find zeros. By one thread,
// after the CTA's last item was taken. stop: a wait ran out.
__device__ __forceinline__ void prompt_leave(const PromptParams& p, int ctas, int stop) {
  if (stop) set_status(p.status, OCCAM_ERR_TIMEOUT);
  if (atomicAdd(&p.counters[1], 1) == ctas - 1) {
    p.counters[0] = 0;
    p.counters[1] = 0;
  }
}

constexpr uint64_t kPromptWaitNs = 2000000000ull;
constexpr uint32_t kPromptTries = 1u << 21;  // of a wait: a second or so
// A bounded wait on a barrier phase; false if it ran out or another role gave up. (Few instructions: the roles together have
// to stay within the instruction cache. What went wrong is recorded when the CTA ends.)
__device__ __forceinline__ bool prompt_wait(uint64_t* bar, uint32_t parity, volatile int* stop) {
  if (__builtin_expect(tc::bar_try(bar, parity), 1)) return true;
  for (uint32_t n = 0; !tc::bar_try(bar, parity); ++n)
    if (n > kPromptTries || *stop) {
      *stop = 1;
      return false;
    }
  return true;
}
#define PROMPT_WAIT(bar, parity) \
  if (__builtin_expect(!prompt_wait(&(bar), (parity), &sh.stop), 0)) return;
// a branch whose code is put out of the way of the loop's
#define PROMPT_RARE(x) __builtin_expect(!!(x), 0)

template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if (BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  return tc::pack_f16(lo, hi);
}

// Tensor map of rows [rows][heads][dim] of 16-bit values, `row` elements apart, as boxes of box_dims dims x
// box_heads x box_rows, swizzled by 64 dims' 128 bytes or 16 dims' 32; dims past the last one are read as zeros.
bool encode_rows(CUtensorMap* m, const void* at, bool bf16, int dim, int heads, int64_t rows, int64_t row, int box_heads,
                 int box_rows, int box_dims = 64);

// Byte offsets of the workspace: the status word (8 bytes) and the counters, zero between calls; then what the
// gradient writes before it reads it (see GradParams).
struct PromptWs {
  size_t terms, stat, norm, power, vnorm, split, total;
};
// How many parts an item of the gradient's keys may be divided into: kPartItems / items, whole, so that nothing is divided
// where there are more than half as many items (tiles x key heads), one an SM or so, and all parts together are kPartItems
// tiles at most, for which the workspace has room. An item would be a CTA's whole time there. (2,400 rows of 28 heads on 4,
// 76 items: 178 us; with parts for 228 items 190, for 608 196. 4,177 of 32 on 8, 264 items, whole 404, in two 424.)
constexpr int kPartItems = 304, kMostParts = 8;
inline int prompt_parts(int64_t items) {
  return items < 1 ? 1 : (int)std::min<int64_t>(std::max<int64_t>(kPartItems / items, 1), kMostParts);
}
inline PromptWs prompt_ws(int64_t total_rows, int64_t total_keys, int heads, int kv_heads) {
  PromptWs w;
  w.terms = 256;
  w.stat = w.terms + cache_align((size_t)total_rows * heads * 32);
  w.norm = w.stat + cache_align((size_t)total_rows * heads * 8);
  w.power = w.norm + cache_align((size_t)total_rows * heads * 4);
  w.vnorm = w.power + cache_align((size_t)total_rows * kv_heads * 4);
  w.split = w.vnorm + cache_align((size_t)total_keys * kv_heads * 4);
  // (parts x keys is at most kPartItems tiles' keys; never less for more keys or heads: a workspace serves smaller calls)
  const size_t split = std::min<size_t>((size_t)kMostParts * total_keys * kv_heads, kPartItems * 128);
  w.total = w.split + cache_align(split * 2 * 128 * 4);
  return w;
}

// Checks the arguments and fills in what both entry points share.
int prompt_params(const occam_prompt_args* a, void* workspace, size_t workspace_bytes, PromptParams* p);
// Whether a result (of 16-bit elements) shares memory with q, k or v.
bool prompt_meets_inputs(const occam_prompt_args* a, const Extent& x);

}  // namespace occam
