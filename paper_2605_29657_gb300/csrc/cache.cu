// cache.cu -- the paged 8-bit cache: occam_cache_append and the page calls
// (extend, fork, compact, release). The page bookkeeping is a one-CTA kernel
// per call: reference counts are scanned for free pages (lowest first) and
// handed out in call order by prefix sums, so page indices do not depend on
// timing. The codes move in grid-wide kernels behind it. Each bookkeeping kernel is a
// chain of dependent loads and block scans: 3 (release) to 7 us for tens of
// sequences, whose starts overlap the kernel before.
#include <algorithm>
#include <utility>

#include "append.cuh"
#include "nvtx.cuh"

using namespace occam;

int occam::cache_sms() {
  constexpr int kMaxDevices = 64;
  static int sms[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 148;
  if (sms[dev] == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 148;
    sms[dev] = n;  // the same value from every thread
  }
  return sms[dev];
}

namespace {

constexpr int kPlanThreads = 1024;

// ---------------------------------------------------------------- append
// One CTA per (touched page, head, K or V): the new rows' values of the block
// stay in registers between the block's maximum and the rounding, so they are
// read once. Bound by HBM (2 bytes read and 1 written a value): 20 k rows of 32 heads of
// 128 dims take 86 us, 5.8 TB/s (66 % DRAM, 71 % issue active). Four heads a CTA with the next head's rows
// under way measured slower (156 us where one took 121): fewer CTAs fit an SM. One
// row each of 64 sequences takes 10 us, the chain of dependent loads (offsets,
// table, rows, scale).
// MAXV: 8-value vectors a thread holds of a block (128 threads; page_tokens * D / 8 / 128 at most).
// grid: x over (head, K or V), y and z over slots.
// (20 k rows, 64 tokens x 128 dims a block: nine CTAs an SM 85 us, eight 90, ten 95, 256 threads
// a CTA 111. 128 x 128 values a block have no bound: 160 registers and three CTAs an SM, 136 us of 20 k rows;
// bounds of four, five and six gave 115, 105 and 105.)
template <bool BF16, int D, int MAXV>
__global__ void __launch_bounds__(128, MAXV == 8 ? 9 : 1) append_kernel(AppendParams p) {
  __shared__ float r[4];
  pdl_wait();
  const int refused = p.c.status[1] & kRefused;  // (no CTA of this launch sets it)
  const int T = p.c.T, H = p.c.heads;
  const int kv = blockIdx.x & 1, h = (int)(blockIdx.x >> 1);
  const int64_t w = (int64_t)blockIdx.z * gridDim.y + blockIdx.y;
  if (w == 1 && blockIdx.x == 0) record_backward(p);  // (an early CTA, and idle where every sequence has a token)
  const int i = slot_sequence(p.row_off, p.n, p.c.log2T, w);
  const int64_t r0 = p.row_off[i], r1 = p.row_off[i + 1];
  const int64_t local = w - ((r0 >> p.c.log2T) + 2 * (int64_t)i);
  const int seq = p.seqs[i];
  int len = -1;
  if ((unsigned)seq < (unsigned)p.c.max_seqs) len = p.c.length[seq];
  if (refused) return;
  if (local < 0 && r0 <= p.total_rows) return;  // rows before row_off[0] belong to no sequence
  const bool good = r0 >= 0 && r1 >= r0 && r1 <= p.total_rows && len >= r1 - r0 &&
                    len <= (int64_t)p.c.max_pages * T;
  if (!good) {
    if (threadIdx.x == 0) set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
    return;
  }
  const int start = len - (int)(r1 - r0);  // position of row r0
  if (local > (len >> p.c.log2T)) return;  // (a slot past the rows)
  const int slot = (start >> p.c.log2T) + (int)local;
  if (slot >= p.c.max_pages) return;
  const int t0 = max(start - slot * T, 0), t1 = min(len - slot * T, T);  // new tokens of this page
  if (t1 <= t0) return;
  if (!in_bounds(i >= 0 && i < p.n && r0 + (int64_t)slot * T - start + t0 >= r0 && r0 + (int64_t)slot * T - start + t1 <= r1,
                 p.c.status, kSiteAppendRow))
    return;
  const int page = p.c.table[(int64_t)seq * p.c.max_pages + slot];
  if ((unsigned)page >= (unsigned)p.c.pages) {
    if (threadIdx.x == 0) set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
    return;
  }
  const int holders = p.c.refs[page];
  const int64_t block = ((int64_t)p.layer * p.c.pages + page) * H;
  const int64_t ld = kv ? p.v_row : p.k_row;
  constexpr int vpr = D / 8;  // vectors of a row
  const int nv = (t1 - t0) * vpr, tv = threadIdx.x / vpr, c = threadIdx.x % vpr;
  const uint16_t* src = static_cast<const uint16_t*>(kv ? p.v : p.k) + (r0 + (int64_t)slot * T - start + t0 + tv) * ld + c * 8;
  const int64_t step = 128 / vpr * ld;
  uint4 x[MAXV];
#pragma unroll
  for (int q = 0; q < MAXV; ++q)
    if (q * 128 + (int)threadIdx.x < nv) x[q] = ldg_stream(src + q * step + h * D);
  if (holders != 1) {  // other sequences hold the page (the same in every thread)
    if (threadIdx.x == 0) set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
    return;
  }
  uint8_t* codes = (kv ? p.c.v : p.c.k) + (block + h) * T * D;
  float* scale = (kv ? p.c.v_scale : p.c.k_scale) + block + h;
  float amax = 0.f;
#pragma unroll
  for (int q = 0; q < MAXV; ++q)
    if (q * 128 + (int)threadIdx.x < nv) amax = fmaxf(amax, amax8<BF16>(x[q]));
  amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax)));
  if ((threadIdx.x & 31) == 0) r[threadIdx.x >> 5] = amax;
  const float was = t0 > 0 ? *scale : 0.f;
  __syncthreads();  // (and every thread has `was`)
  const float need = block_scale(fmaxf(fmaxf(r[0], r[1]), fmaxf(r[2], r[3])));
  const float now = was > need ? was : need;  // older tokens keep at least their scale
  if (t0 > 0 && now > was) {
    // the held codes, rounded again to the larger scale
    const float ratio = was / now;
    for (int e = threadIdx.x; e < t0 * D / 16; e += 128) {
      uint4 y = reinterpret_cast<uint4*>(codes)[e];
      uint32_t* rw = reinterpret_cast<uint32_t*>(&y);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float f[4];
        codes4_f32(rw[j], f);
#pragma unroll
        for (int m = 0; m < 4; ++m) f[m] *= ratio;
        rw[j] = f32_codes4(f);
      }
      reinterpret_cast<uint4*>(codes)[e] = y;
    }
  }
  const bool exact = is_pow2(now);
  const float inv = 1.f / now;
#pragma unroll
  for (int q = 0; q < MAXV; ++q) {
    if (q * 128 + (int)threadIdx.x < nv)
      *reinterpret_cast<uint2*>(codes + (t0 + tv + q * (128 / vpr)) * D + c * 8) =
          exact ? codes8<BF16>(x[q], inv) : codes8_by_division<BF16>(x[q], now);
  }
  if (threadIdx.x == 0) *scale = now;
}

// ---------------------------------------------------------------- page bookkeeping (one CTA)

// The slots a call names, a bit each.
constexpr int kSlotWords = 65536 / 32;
// (before the kernel waits for the one before it)
__device__ __forceinline__ void clear_slots(const CacheDev& c, uint32_t* bits) {
  for (int i = threadIdx.x; i < (c.max_seqs + 31) / 32; i += blockDim.x) bits[i] = 0;
  __syncthreads();
}
// Marks the n slots of `seqs`; true (block-wide) if all are in range and listed once.
__device__ bool mark_slots(const CacheDev& c, const int32_t* seqs, int n, uint32_t* bits) {
  int bad = 0;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int s = seqs[i];
    const uint32_t bit = 1u << (s & 31);
    if ((unsigned)s >= (unsigned)c.max_seqs || (atomicOr(&bits[s >> 5], bit) & bit)) bad = 1;
  }
  return __syncthreads_or(bad) == 0;
}

// The block's sum, to every thread. A call's page counts are added in 64 bits (a sequence may want
// up to 2^27 pages); once the sum is known to fit the pool, 32 bits do. tmp: 32 words of shared memory.
__device__ int64_t block_sum(int64_t x, int64_t* tmp) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) tmp[threadIdx.x >> 5] = x;
  __syncthreads();
  int64_t sum = 0;
  for (int w = 0; w < kPlanThreads / 32; ++w) sum += tmp[w];
  __syncthreads();
  return sum;
}

// Writes the lowest `want` free pages, ascending, to list; returns how many
// there are (want, 0 .. c.pages, or fewer if the pool has fewer). tmp: 33 ints of shared memory.
__device__ int find_free(const CacheDev& c, int want, int32_t* list, int* tmp) {
  int found = 0;
  const bool vec = (reinterpret_cast<uintptr_t>(c.refs) & 15) == 0;
  for (int base = 0; base < c.pages && found < want; base += 4 * kPlanThreads) {
    const int p = base + 4 * threadIdx.x;
    int r[4] = {1, 1, 1, 1};
    if (vec && p + 4 <= c.pages) {
      const int4 q = *reinterpret_cast<const int4*>(c.refs + p);
      r[0] = q.x;
      r[1] = q.y;
      r[2] = q.z;
      r[3] = q.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (p + j < c.pages) r[j] = c.refs[p + j];
    }
    int f = 0, total = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) f += r[j] == 0;
    int at = found + block_exclusive_scan(f, tmp, &total);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (r[j] == 0) {
        if (at < want && in_bounds(at >= 0 && at < c.pages, c.status, kSiteFreeList)) list[at] = p + j;
        ++at;
      }
    found += total;
  }
  __syncthreads();  // the list is complete for every thread of the block
  return min(found, want);
}

struct PlanParams {
  CacheDev c;
  int n;
  const int32_t* a;  // extend: seqs; fork: src; compact: seqs
  const int32_t* b;  // extend: counts; fork: dst
  int32_t* free_list;
  int2* new_pages;   // fork: (from, to) of a copied page, or (-1, -1)
  // compact
  int32_t* count;
  int32_t* lead;
  int32_t* head;
  int32_t* old_table;
};

__device__ __forceinline__ int pages_of(int tokens, const CacheDev& c) { return (tokens + c.T - 1) >> c.log2T; }

__global__ void __launch_bounds__(kPlanThreads) extend_kernel(PlanParams p) {
  __shared__ int tmp[33];
  __shared__ int64_t sums[32];
  __shared__ uint32_t slots[kSlotWords];
  clear_slots(p.c, slots);
  pdl_wait();
  const CacheDev& c = p.c;
  if (c.status[1] & kRefused) return;
  const bool fine = mark_slots(c, p.a, p.n, slots);
  int bad = 0, full = 0;
  int64_t total = 0;
  if (fine) {
    for (int i = threadIdx.x; i < p.n; i += kPlanThreads) {
      const int s = p.a[i], add = p.b[i], len = c.length[s];
      const int64_t to = (int64_t)len + add;
      if (add < 0 || len < 0 || len > c.max_pages * c.T) {
        bad = 1;
      } else if (to > (int64_t)c.max_pages * c.T) {
        full = 1;
      } else {
        total += pages_of((int)to, c) - pages_of(len, c);
        // tokens go into a page of the sequence's own
        if (add > 0 && (len & (c.T - 1))) {
          const int pg = c.table[(int64_t)s * c.max_pages + (len >> c.log2T)];
          if ((unsigned)pg >= (unsigned)c.pages || c.refs[pg] != 1) bad = 1;
        }
      }
    }
  }
  total = block_sum(total, sums);
  bad = __syncthreads_or(bad || !fine);
  full = __syncthreads_or(full) || total > c.pages;
  const bool ok = !bad && !full && find_free(c, (int)total, p.free_list, tmp) == (int)total;
  if (ok) {
    int at = 0;
    for (int base = 0; base < p.n; base += kPlanThreads) {
      const int i = base + threadIdx.x;
      int need = 0, have = 0, s = 0, t = 0, to = 0;
      if (i < p.n) {
        s = p.a[i];
        const int len = c.length[s];
        to = len + p.b[i];
        have = pages_of(len, c);
        need = pages_of(to, c) - have;
      }
      int rank = at + block_exclusive_scan(need, tmp, &t);
      at += t;
      for (int j = 0; j < need; ++j) {
        if (!in_bounds(rank >= 0 && rank + j < c.pages && have + j < c.max_pages, c.status, kSiteFreeList)) break;
        const int pg = p.free_list[rank + j];
        if (!in_bounds((unsigned)pg < (unsigned)c.pages, c.status, kSiteTable)) break;
        c.table[(int64_t)s * c.max_pages + have + j] = pg;
        c.refs[pg] = 1;
      }
      if (i < p.n) c.length[s] = to;
    }
  } else if (threadIdx.x == 0) {
    set_status(c.status, bad ? OCCAM_ERR_INVALID_ARG : OCCAM_ERR_CAPACITY);
    atomicOr(&c.status[1], kRefused);
  }
}

__global__ void __launch_bounds__(kPlanThreads) fork_kernel(PlanParams p) {
  __shared__ int tmp[33];
  __shared__ uint32_t slots[kSlotWords];
  clear_slots(p.c, slots);
  pdl_wait();
  const CacheDev& c = p.c;
  const bool fine = mark_slots(c, p.b, p.n, slots);
  int bad = 0;
  int64_t total = 0;
  if (fine) {
    for (int base = 0; base < p.n; base += kPlanThreads) {
      const int i = base + threadIdx.x;
      int need = 0, t = 0;
      if (i < p.n) {
        const int a = p.a[i], b = p.b[i];
        p.new_pages[i] = make_int2(-1, -1);
        if ((unsigned)a >= (unsigned)c.max_seqs || ((slots[a >> 5] >> (a & 31)) & 1) || c.length[b] != 0 || c.length[a] < 0 ||
            c.length[a] > c.max_pages * c.T)
          bad = 1;
        else
          need = (c.length[a] & (c.T - 1)) != 0;
      }
      block_exclusive_scan(need, tmp, &t);
      total += t;
    }
    // every page that is shared or copied must be one
    if (!__syncthreads_or(bad)) {
      const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
      for (int i = warp; i < p.n; i += kPlanThreads / 32) {
        const int a = p.a[i], m = pages_of(c.length[a], c);
        for (int j = lane; j < m; j += 32)
          if ((unsigned)c.table[(int64_t)a * c.max_pages + j] >= (unsigned)c.pages) bad = 1;
      }
    }
  }
  bad = __syncthreads_or(bad || !fine);
  const bool ok = !bad && total <= c.pages && find_free(c, (int)total, p.free_list, tmp) == (int)total;
  if (ok) {
    int at = 0;
    for (int base = 0; base < p.n; base += kPlanThreads) {
      const int i = base + threadIdx.x;
      int need = 0, t = 0, a = 0, b = 0, len = 0;
      if (i < p.n) {
        a = p.a[i];
        b = p.b[i];
        len = c.length[a];
        need = (len & (c.T - 1)) != 0;
      }
      const int rank = at + block_exclusive_scan(need, tmp, &t);
      at += t;
      if (need && in_bounds(rank >= 0 && rank < c.pages && (len >> c.log2T) < c.max_pages, c.status, kSiteFreeList) &&
          in_bounds((unsigned)p.free_list[rank] < (unsigned)c.pages, c.status, kSiteTable)) {
        const int pg = p.free_list[rank], j = len >> c.log2T;
        p.new_pages[i] = make_int2(c.table[(int64_t)a * c.max_pages + j], pg);
        c.table[(int64_t)b * c.max_pages + j] = pg;
        c.refs[pg] = 1;
      }
      if (i < p.n) c.length[b] = len;
    }
    // full pages are shared: a warp per pair
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = warp; i < p.n; i += kPlanThreads / 32) {
      const int a = p.a[i], b = p.b[i], m = c.length[a] >> c.log2T;
      for (int j = lane; j < m; j += 32) {
        const int pg = c.table[(int64_t)a * c.max_pages + j];
        if (!in_bounds((unsigned)pg < (unsigned)c.pages && j < c.max_pages, c.status, kSiteTable)) break;
        c.table[(int64_t)b * c.max_pages + j] = pg;
        atomicAdd(&c.refs[pg], 1);
      }
    }
  } else {
    for (int i = threadIdx.x; i < p.n; i += blockDim.x) p.new_pages[i] = make_int2(-1, -1);
    if (threadIdx.x == 0) set_status(c.status, bad ? OCCAM_ERR_INVALID_ARG : OCCAM_ERR_CAPACITY);
  }
}

// Copies the pages fork_kernel listed: grid (pairs, layers, 2 * chunks), 16 KB a CTA.
constexpr int kCopyChunk = 16384;
__global__ void __launch_bounds__(256) copy_pages_kernel(CacheDev c, const int2* pairs, int page_bytes) {
  pdl_wait();
  const int2 ft = pairs[blockIdx.x];
  if (ft.x < 0) return;
  if (!in_bounds(ft.x < c.pages && (unsigned)ft.y < (unsigned)c.pages, c.status, kSiteCopyPage)) return;
  const int layer = blockIdx.y, kv = blockIdx.z & 1, chunk = blockIdx.z >> 1;
  const int64_t from = (int64_t)layer * c.pages + ft.x, to = (int64_t)layer * c.pages + ft.y;
  uint8_t* base = kv ? c.v : c.k;
  const uint4* src = reinterpret_cast<const uint4*>(base + from * page_bytes);
  uint4* dst = reinterpret_cast<uint4*>(base + to * page_bytes);
  const int e0 = chunk * (kCopyChunk / 16) + threadIdx.x, n = page_bytes / 16;
  uint4 x[4];
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (e0 + q * 256 < n) x[q] = ldg_stream(src + e0 + q * 256);
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (e0 + q * 256 < n) stg_stream(dst + e0 + q * 256, x[q]);
  if (chunk == 0) {
    float* sc = kv ? c.v_scale : c.k_scale;
    for (int h = threadIdx.x; h < c.heads; h += 256) sc[to * c.heads + h] = sc[from * c.heads + h];
  }
}

__global__ void __launch_bounds__(256) release_kernel(CacheDev c, int n, const int32_t* seqs) {
  pdl_wait();
  const int i = blockIdx.y;
  const int s = seqs[i];
  if ((unsigned)s >= (unsigned)c.max_seqs) {
    if (threadIdx.x == 0 && blockIdx.x == 0) set_status(c.status, OCCAM_ERR_INVALID_ARG);
    return;
  }
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j < c.max_pages) {
    // taking the entry makes a slot listed twice give its pages back once
    int32_t* e = &c.table[(int64_t)s * c.max_pages + j];
    if (*e != -1) {
      const int pg = atomicExch(e, -1);
      if (pg != -1) {
        if ((unsigned)pg >= (unsigned)c.pages)
          set_status(c.status, OCCAM_ERR_INVALID_ARG);
        else
          atomicSub(&c.refs[pg], 1);
      }
    }
  }
  if (j == 0) c.length[s] = 0;
}

// ---------------------------------------------------------------- compact
struct CountParams {
  CacheDev c;
  const int32_t* seqs;
  const uint8_t* keep;
  const int64_t* keep_off;
  int64_t total_keep;
  int32_t* count;
  int32_t* lead;
  int2* info;  // (listed tokens, flags)
  int32_t* list;
};

// One CTA per sequence: the positions of its kept flagged tokens, in order, to
// list[keep_off[i] ..], their number and the number of leading full pages
// that keep every token. count = -1 marks bad offsets.
__global__ void __launch_bounds__(1024) compact_count_kernel(CountParams p) {
  __shared__ int tmp[33];
  __shared__ int first;
  pdl_wait();
  const int i = blockIdx.x;
  const int s = p.seqs[i];
  const int64_t k0 = p.keep_off[i], k1 = p.keep_off[i + 1];
  const int len = (unsigned)s < (unsigned)p.c.max_seqs ? p.c.length[s] : -1;
  if (len < 0 || len > p.c.max_pages * p.c.T || k0 < 0 || k1 < k0 || k1 > p.total_keep) {
    if (threadIdx.x == 0) p.count[i] = -1;
    return;
  }
  const int flags = (int)(k1 - k0 < len ? k1 - k0 : len);
  if (threadIdx.x == 0) first = len;  // first dropped position
  __syncthreads();
  int n = 0, mine = len;
  for (int base = 0; base < flags; base += 1024) {
    const int pos = base + threadIdx.x;
    const int k = pos < flags && in_bounds(k0 + pos < p.total_keep, p.c.status, kSiteKeepList) && p.keep[k0 + pos] != 0;
    if (pos < flags && !k) mine = min(mine, pos);
    int t = 0;
    const int at = n + block_exclusive_scan(k, tmp, &t);
    if (k && in_bounds(k0 + at < p.total_keep, p.c.status, kSiteKeepList)) p.list[k0 + at] = pos;
    n += t;
  }
  mine = __reduce_min_sync(0xffffffffu, mine);
  if ((threadIdx.x & 31) == 0) atomicMin(&first, mine);
  __syncthreads();
  if (threadIdx.x == 0) {
    p.count[i] = n + (len - flags);  // tokens past the flags stay
    p.info[i] = make_int2(n, flags);
    p.lead[i] = first >> p.c.log2T;
  }
}

// New page tables: head[i] = index of sequence i's first new page in free_list.
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(PlanParams p) {
  __shared__ int tmp[33];
  __shared__ int64_t sums[32];
  __shared__ uint32_t slots[kSlotWords];
  clear_slots(p.c, slots);
  pdl_wait();
  const CacheDev& c = p.c;
  const bool fine = mark_slots(c, p.a, p.n, slots);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int bad = 0;
  int64_t total = 0;
  auto pages_wanted = [&](int i) { return max(pages_of(p.count[i], c) - p.lead[i], 0); };
  if (fine) {
    for (int i = threadIdx.x; i < p.n; i += kPlanThreads) {
      if (p.count[i] < 0)
        bad = 1;
      else
        total += pages_wanted(i);
    }
  }
  total = block_sum(total, sums);
  if (fine && !__syncthreads_or(bad) && total <= c.pages) {
    for (int i = warp; i < p.n; i += kPlanThreads / 32) {
      const int s = p.a[i], m = pages_of(c.length[s], c);
      for (int j = lane; j < m; j += 32)
        if ((unsigned)c.table[(int64_t)s * c.max_pages + j] >= (unsigned)c.pages) bad = 1;
    }
  }
  bad = __syncthreads_or(bad || !fine);
  const bool ok = !bad && total <= c.pages && find_free(c, (int)total, p.free_list, tmp) == (int)total;
  if (ok) {
    for (int base = 0, at = 0; base < p.n; base += kPlanThreads) {
      const int i = base + threadIdx.x;
      int sum = 0;
      const int before = at + block_exclusive_scan(i < p.n ? pages_wanted(i) : 0, tmp, &sum);
      if (i < p.n) p.head[i] = before;
      at += sum;
    }
    __syncthreads();
    // pages leave their sequence before new ones come in: the new ones were
    // free at the start of the call, so the two sets do not meet
    for (int i = warp; i < p.n; i += kPlanThreads / 32) {
      const int s = p.a[i], lead = p.lead[i], m = pages_of(c.length[s], c);
      const int to = pages_of(p.count[i], c), head = p.head[i];
      for (int j = lane; j < max(m, to); j += 32) {
        int32_t* e = &c.table[(int64_t)s * c.max_pages + j];
        if (!in_bounds(j < c.max_pages && (j < lead || j >= to || (unsigned)(head + j - lead) < (unsigned)c.pages), c.status,
                       kSiteFreeList))
          break;
        if (j < m) {
          const int pg = *e;
          if (!in_bounds((unsigned)pg < (unsigned)c.pages, c.status, kSiteTable)) break;
          p.old_table[(int64_t)i * c.max_pages + j] = pg;
          if (j >= lead) atomicSub(&c.refs[pg], 1);
        }
        if (j >= lead) {
          const bool fresh = j < to;
          const int pg = fresh ? p.free_list[head + j - lead] : -1;
          if (!in_bounds(!fresh || (unsigned)pg < (unsigned)c.pages, c.status, kSiteTable)) break;
          *e = pg;
          if (fresh) atomicAdd(&c.refs[pg], 1);
        }
      }
      __syncwarp();
      if (lane == 0) c.length[s] = p.count[i];
    }
    if (threadIdx.x == 0) p.head[p.n] = (int)total;
  } else {
    if (threadIdx.x == 0) {
      p.head[p.n] = 0;  // nothing to move
      set_status(c.status, bad ? OCCAM_ERR_INVALID_ARG : OCCAM_ERR_CAPACITY);
    }
  }
}

// the largest |code| of 16 (NaN codes passed over): magnitudes order as integers
__device__ __forceinline__ float codes_amax(uint4 v) {
  const uint32_t w[4] = {v.x & 0x7f7f7f7fu, v.y & 0x7f7f7f7fu, v.z & 0x7f7f7f7fu, v.w & 0x7f7f7f7fu};
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t nan = __vcmpeq4(w[k], 0x7f7f7f7fu);
    m = __vmaxu4(m, w[k] & ~nan);
  }
  m = __vmaxu4(m, m >> 16);
  m = max(m & 0xffu, m >> 8 & 0xffu);
  float f[4];
  codes4_f32(m, f);
  return f[0];
}

struct MoveParams {
  CacheDev c;
  int n, layer0, layers;
  const int32_t* free_list;
  const int32_t* head;
  const int32_t* lead;
  const int32_t* count;
  const int32_t* old_table;
  const int2* info;
  const int32_t* list;
  const int64_t* keep_off;
};

// One CTA per (new page, layer, K or V, group of heads), a block of codes at
// a time: the kept rows are gathered once, their common scale found, the codes
// rounded to it (a shift of the exponent where both scales are powers of
// two) and written once. 8 x 350 scattered rows of 2 x 32 heads in 11 layers take 95 to 102 us, 4.5 TB/s of
// bytes moved, at 56 % DRAM and 59 % issue active with 48 % of the warps: bound by neither alone, but
// by a head's chain (loads, maximum across a barrier, stores) before the next head's loads.
// MAXV: 16-code vectors a thread holds (128 threads).
constexpr int kMoveHeads = 4;
// A code times its scale may round to 2^128 (256 x 2^120, from values near bf16's end): it counts as the
// largest finite value, which asks for the same scale.
constexpr float kLargest = 3.4028235e38f;
template <int D, int MAXV>
__global__ void __launch_bounds__(128) compact_move_kernel(MoveParams p) {
  __shared__ int2 src[128];  // page and slot of each token
  __shared__ float red[2][4];
  pdl_wait();
  constexpr int vpr = D / 16;
  const int T = p.c.T, H = p.c.heads;
  const int hg = (H + kMoveHeads - 1) / kMoveHeads, per_page = p.layers * 2 * hg;
  const int pages = p.head[p.n];
  const int tv = threadIdx.x / vpr, c = threadIdx.x % vpr;
  for (int fresh = blockIdx.y; fresh < pages; fresh += gridDim.y) {
    // the sequence whose new pages include this one (head is ascending)
    int lo = 0, hi = p.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.head[mid] <= fresh) lo = mid; else hi = mid;
    }
    const int i = lo;
    const int first = (p.lead[i] + fresh - p.head[i]) * T;  // new position of the page's first token
    const int tokens = min(p.count[i] - first, T), nv = tokens * vpr;
    __syncthreads();
    bool fits = in_bounds(i < p.n && fresh < p.c.pages && (unsigned)p.free_list[fresh] < (unsigned)p.c.pages, p.c.status, kSiteMoveToken);
    if (fits && (int)threadIdx.x < tokens) {
      // kept flagged tokens come from the list, tokens past the flags in order
      const int q = first + threadIdx.x;
      const int2 info = p.info[i];  // listed tokens, flags
      const bool listed = in_bounds(q >= info.x || p.keep_off[i] + q < p.keep_off[i + 1], p.c.status, kSiteKeepList);
      const int pos = q < info.x && listed ? p.list[p.keep_off[i] + q] : info.y + q - info.x;
      fits = listed && in_bounds(pos >= 0 && (pos >> p.c.log2T) < p.c.max_pages, p.c.status, kSiteMoveToken);
      const int page = fits ? p.old_table[(int64_t)i * p.c.max_pages + (pos >> p.c.log2T)] : 0;
      fits = fits && in_bounds((unsigned)page < (unsigned)p.c.pages, p.c.status, kSiteMoveToken);
      src[threadIdx.x] = make_int2(page, pos & (T - 1));
    }
    __syncthreads();
#if OCCAM_CHECKED
    if (!__syncthreads_and(fits)) continue;
#endif
    const int to_page = p.free_list[fresh];
    for (int item = blockIdx.x; item < per_page; item += gridDim.x) {
      const int g = item % hg, kv = item / hg & 1, layer = p.layer0 + item / hg / 2;
      const int h0 = g * kMoveHeads, h1 = min(h0 + kMoveHeads, H);
      uint8_t* codes = kv ? p.c.v : p.c.k;
      float* sc = kv ? p.c.v_scale : p.c.k_scale;
      const int64_t layer_page = (int64_t)layer * p.c.pages, new_block = (layer_page + to_page) * H;
      // this thread's vectors: block of head 0, and the place in it
      int64_t from[MAXV];
      int at[MAXV];
#pragma unroll
      for (int q = 0; q < MAXV; ++q) {
        const int2 ps = src[min(tv + q * (128 / vpr), 127)];
        from[q] = (layer_page + ps.x) * H;
        at[q] = ps.y * D + c * 16;
      }
      auto load = [&](uint4 (&x)[MAXV], float (&s)[MAXV], int h) {
#pragma unroll
        for (int q = 0; q < MAXV; ++q)
          if (q * 128 + (int)threadIdx.x < nv) {
            x[q] = ldg_stream(codes + (from[q] + h) * T * D + at[q]);
            s[q] = sc[from[q] + h];
          }
      };
      auto finish = [&](uint4 (&x)[MAXV], const float (&s)[MAXV], int h) {
        float amax = 0.f;
#pragma unroll
        for (int q = 0; q < MAXV; ++q)
          if (q * 128 + (int)threadIdx.x < nv) amax = fmaxf(amax, fminf(codes_amax(x[q]) * s[q], kLargest));
        amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax)));
        float* r = red[h & 1];
        if ((threadIdx.x & 31) == 0) r[threadIdx.x >> 5] = amax;
        __syncthreads();
        const float now = block_scale(fmaxf(fmaxf(r[0], r[1]), fmaxf(r[2], r[3])));
        const float inv = 1.f / now;  // exact: now is a power of two
        uint8_t* out = codes + (new_block + h) * T * D;
#pragma unroll
        for (int q = 0; q < MAXV; ++q) {
          if (q * 128 + (int)threadIdx.x < nv) {
            uint32_t* w = reinterpret_cast<uint32_t*>(&x[q]);
            if (s[q] != now) {
              // (finite, so that a code of 0 stays 0 under any scale)
              const float ratio = fminf(s[q] * inv, 3.4e38f);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                float f[4];
                codes4_f32(w[j], f);
#pragma unroll
                for (int k = 0; k < 4; ++k) f[k] *= ratio;
                w[j] = f32_codes4(f);
              }
            }
            stg_stream(out + (q * 128 + threadIdx.x) * 16, x[q]);
          }
        }
        if (threadIdx.x == 0) sc[new_block + h] = now;
      };
      for (int h = h0; h < h1; ++h) {
        uint4 x[MAXV];
        float s[MAXV];
        load(x, s, h);
        finish(x, s, h);
      }
      __syncthreads();  // (red: an odd number of heads meets the next item's first)
    }
  }
}

int last_error() { return cudaGetLastError() == cudaSuccess ? OCCAM_OK : OCCAM_ERR_CUDA; }

PlanParams plan_params(const occam_cache* c, void* ws, const CacheWs& w, int n) {
  PlanParams p{};
  p.c = cache_dev(c, ws, w);
  p.n = n;
  p.free_list = ws_at<int32_t>(ws, w.free_list);
  p.new_pages = ws_at<int2>(ws, w.new_pages);
  p.count = ws_at<int32_t>(ws, w.count);
  p.lead = ws_at<int32_t>(ws, w.lead);
  p.head = ws_at<int32_t>(ws, w.head);
  p.old_table = ws_at<int32_t>(ws, w.old_table);
  return p;
}

template <bool BF16, int D>
bool launch_append(AppendParams& p, cudaStream_t st) {
  const int64_t slots = p.total_rows / p.c.T + 2 * (int64_t)p.n;
  const unsigned y = (unsigned)std::min<int64_t>(slots, 65535);
  const dim3 grid((unsigned)p.c.heads * 2, y, (unsigned)((slots + y - 1) / y));
  const int vecs = p.c.T * D / 8 / 128;
  if (vecs <= 2) return launch_after(append_kernel<BF16, D, 2>, grid, 128, 0, st, p);
  if (vecs == 4) return launch_after(append_kernel<BF16, D, 4>, grid, 128, 0, st, p);
  if (vecs == 8) return launch_after(append_kernel<BF16, D, 8>, grid, 128, 0, st, p);
  return launch_after(append_kernel<BF16, D, 16>, grid, 128, 0, st, p);
}

template <int D>
bool launch_move(const MoveParams& m, cudaStream_t st) {
  const int vecs = m.c.T * D / 16 / 128;
  // how many pages move is only known on the device: CTAs share them out, all of a page's work to
  // neighbours
  const int work = m.layers * 2 * ((m.c.heads + kMoveHeads - 1) / kMoveHeads);
  const unsigned x = (unsigned)std::min(work, 65535), want = (unsigned)cache_sms() * 64;
  const dim3 grid(x, std::max(1u, std::min(want / x, 65535u)));
  if (vecs <= 1) return launch_after(compact_move_kernel<D, 1>, grid, 128, 0, st, m);
  if (vecs == 2) return launch_after(compact_move_kernel<D, 2>, grid, 128, 0, st, m);
  if (vecs == 4) return launch_after(compact_move_kernel<D, 4>, grid, 128, 0, st, m);
  return launch_after(compact_move_kernel<D, 8>, grid, 128, 0, st, m);
}

}  // namespace

#define OCCAM_TRY(x)                 \
  do {                               \
    int _rc = (x);                   \
    if (_rc != OCCAM_OK) return _rc; \
  } while (0)

extern "C" {

int occam_cache_workspace_size(const occam_cache* cache, int64_t max_tokens, size_t* bytes) {
  if (!bytes || max_tokens < 0) return OCCAM_ERR_INVALID_ARG;
  OCCAM_TRY(check_cache(cache));
  *bytes = cache_ws(cache, max_tokens).total;
  return OCCAM_OK;
}

int occam_cache_extend(const occam_cache* cache, int32_t n, const int32_t* seqs, const int32_t* counts,
                       void* workspace, size_t workspace_bytes, occam_stream_t stream) {
  const NvtxRange nvtx("occam_cache_extend");
  launch_counter() = 0;
  OCCAM_TRY(check_cache(cache));
  if (n < 0 || n > cache->max_seqs || (n > 0 && (!seqs || !counts))) return OCCAM_ERR_INVALID_ARG;
  CacheWs w;
  OCCAM_TRY(check_cache_ws(cache, 0, workspace, workspace_bytes, &w));
  if (n == 0) return OCCAM_OK;
  PlanParams p = plan_params(cache, workspace, w, n);
  p.a = seqs;
  p.b = counts;
  return launch_after(extend_kernel, dim3(1), kPlanThreads, 0, reinterpret_cast<cudaStream_t>(stream), p)
             ? last_error()
             : OCCAM_ERR_CUDA;
}

int occam_cache_append(const occam_cache* cache, int32_t layer, int32_t dtype, int64_t total_rows, const void* k,
                       int64_t k_row, const void* v, int64_t v_row, int32_t n, const int32_t* seqs,
                       const int64_t* row_off, void* workspace, size_t workspace_bytes, occam_stream_t stream) {
  const NvtxRange nvtx("occam_cache_append");
  launch_counter() = 0;
  OCCAM_TRY(check_cache(cache));
  if (dtype != OCCAM_BF16 && dtype != OCCAM_F16) return OCCAM_ERR_UNSUPPORTED;
  if (layer < 0 || layer >= cache->layers || total_rows < 0 || total_rows > 0x7fffffff || n < 0 || n > cache->max_seqs)
    return OCCAM_ERR_INVALID_ARG;
  CacheWs w;
  OCCAM_TRY(check_cache_ws(cache, 0, workspace, workspace_bytes, &w));
  if (n == 0 || total_rows == 0) return OCCAM_OK;
  const int64_t row = (int64_t)cache->heads * cache->dim;
  if (!k || !v || !seqs || !row_off || !aligned16(k) || !aligned16(v) || k_row < row || v_row < row || (k_row & 7) || (v_row & 7))
    return OCCAM_ERR_INVALID_ARG;
  AppendParams p{};
  p.c = cache_dev(cache, workspace, w);
  p.layer = layer;
  p.n = n;
  p.total_rows = total_rows;
  p.k_row = k_row;
  p.v_row = v_row;
  p.k = k;
  p.v = v;
  p.seqs = seqs;
  p.row_off = row_off;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const bool bf16 = dtype == OCCAM_BF16;
  const bool ok = cache->dim == 128 ? (bf16 ? launch_append<true, 128>(p, st) : launch_append<false, 128>(p, st))
                                    : (bf16 ? launch_append<true, 64>(p, st) : launch_append<false, 64>(p, st));
  return ok ? last_error() : OCCAM_ERR_CUDA;
}

int occam_cache_fork(const occam_cache* cache, int32_t n, const int32_t* src, const int32_t* dst, void* workspace,
                     size_t workspace_bytes, occam_stream_t stream) {
  const NvtxRange nvtx("occam_cache_fork");
  launch_counter() = 0;
  OCCAM_TRY(check_cache(cache));
  if (n < 0 || n > cache->max_seqs || (n > 0 && (!src || !dst))) return OCCAM_ERR_INVALID_ARG;
  CacheWs w;
  OCCAM_TRY(check_cache_ws(cache, 0, workspace, workspace_bytes, &w));
  if (n == 0) return OCCAM_OK;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  PlanParams p = plan_params(cache, workspace, w, n);
  p.a = src;
  p.b = dst;
  if (!launch_after(fork_kernel, dim3(1), kPlanThreads, 0, st, p)) return OCCAM_ERR_CUDA;
  const int page_bytes = cache->heads * cache->page_tokens * cache->dim;
  const int chunks = (page_bytes + kCopyChunk - 1) / kCopyChunk;
  const dim3 grid((unsigned)n, (unsigned)cache->layers, (unsigned)(2 * chunks));
  return launch_after(copy_pages_kernel, grid, 256, 0, st, p.c, p.new_pages, page_bytes) ? last_error() : OCCAM_ERR_CUDA;
}

int occam_cache_compact(const occam_cache* cache, int32_t layer_begin, int32_t layer_end, int32_t n,
                        const int32_t* seqs, const uint8_t* keep, const int64_t* keep_off, int64_t total_keep,
                        void* workspace, size_t workspace_bytes, occam_stream_t stream) {
  const NvtxRange nvtx("occam_cache_compact");
  launch_counter() = 0;
  OCCAM_TRY(check_cache(cache));
  if (layer_begin < 0 || layer_end < layer_begin || layer_end > cache->layers || n < 0 || n > cache->max_seqs ||
      total_keep < 0 || (n > 0 && (!seqs || !keep_off)) || (total_keep > 0 && !keep))
    return OCCAM_ERR_INVALID_ARG;
  CacheWs w;
  OCCAM_TRY(check_cache_ws(cache, total_keep, workspace, workspace_bytes, &w));
  if (n == 0) return OCCAM_OK;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  PlanParams p = plan_params(cache, workspace, w, n);
  p.a = seqs;
  CountParams q{};
  q.c = p.c;
  q.seqs = seqs;
  q.keep = keep;
  q.keep_off = keep_off;
  q.total_keep = total_keep;
  q.count = p.count;
  q.lead = p.lead;
  q.info = p.new_pages;
  q.list = ws_at<int32_t>(workspace, w.list);
  if (!launch_after(compact_count_kernel, dim3((unsigned)n), 1024, 0, st, q) ||
      !launch_after(compact_plan_kernel, dim3(1), kPlanThreads, 0, st, p))
    return OCCAM_ERR_CUDA;
  if (layer_end > layer_begin) {
    MoveParams m{};
    m.c = p.c;
    m.n = n;
    m.layer0 = layer_begin;
    m.layers = layer_end - layer_begin;
    m.free_list = p.free_list;
    m.head = p.head;
    m.lead = p.lead;
    m.count = p.count;
    m.old_table = p.old_table;
    m.info = p.new_pages;
    m.list = q.list;
    m.keep_off = keep_off;
    if (!(cache->dim == 128 ? launch_move<128>(m, st) : launch_move<64>(m, st))) return OCCAM_ERR_CUDA;
  }
  return last_error();
}

int occam_cache_release(const occam_cache* cache, int32_t n, const int32_t* seqs, void* workspace,
                        size_t workspace_bytes, occam_stream_t stream) {
  const NvtxRange nvtx("occam_cache_release");
  launch_counter() = 0;
  OCCAM_TRY(check_cache(cache));
  if (n < 0 || n > cache->max_seqs || (n > 0 && !seqs)) return OCCAM_ERR_INVALID_ARG;
  CacheWs w;
  OCCAM_TRY(check_cache_ws(cache, 0, workspace, workspace_bytes, &w));
  if (n == 0) return OCCAM_OK;
  const dim3 grid((unsigned)((cache->max_pages + 255) / 256), (unsigned)n);
  return launch_after(release_kernel, grid, 256, 0, reinterpret_cast<cudaStream_t>(stream), cache_dev(cache, workspace, w), n, seqs)
             ? last_error()
             : OCCAM_ERR_CUDA;
}

}  // extern "C"
