// attend_shared.cu -- attention of sequences that share leading pages (forks of
// one prefix): occam_cache_attend_shared.
//
// The softmax over a row's keys is split where its group's common pages end: with
// (o_1, L_1) over the prefix and (o_2, L_2) over the tail, L = log sum exp of the two parts,
//   o = (o_1 e^{L_1} + o_2 e^{L_2}) / (e^{L_1} + e^{L_2}).
// The rows of a group's sequences lie next to one another and all see the whole prefix,
// so over the prefix they are the rows of one sequence: its codes are read once a group and, from 33 rows a
// key head on, multiplied on the tensor cores, instead of once a sequence. Launches:
// how many leading pages the tables of each group have in common (this file), the
// prefixes, the sums of prefixes that were split, then the tails, whose rows take the prefix's result in as they are written
// (attend.cu and attend_tc.cu, as attention over whole sequences).
// What bounds it is the chain of these launches and the parts of split prefixes, not the codes: 64 forks of one token over
// 16,000 common ones (8 key heads of 128, 4 query heads each) take 66 us, where reading the codes once takes 9 and
// each sequence by itself 480.
#include <algorithm>

#include "attend.cuh"
#include "nvtx.cuh"

using namespace occam;

namespace {

constexpr int kThreads = 1024;
constexpr float kChain = 15.f;    // us of the launches that sharing adds
constexpr float kJoin = 0.0005f;  // us of a (row, head) whose two parts are joined

// Row tiles' worth of time that m query rows of a key head take against the same keys
__device__ __forceinline__ float row_tiles(float m) { return m <= 0.f ? 0.f : m <= 32.f ? 0.5f : ceilf(m / 256.f); }

struct SharedWs {
  size_t shared, skip, pre_l, pre_o, ranges, total;
  int64_t range_tiles;
};
// Behind what attention itself uses (where other calls on the same workspace keep their lists: each call writes
// before it reads)
SharedWs shared_ws(const occam_cache* c, int64_t total_rows, int heads) {
  SharedWs w;
  w.shared = cache_ws(c, 0).total;
  w.skip = w.shared + cache_align((size_t)c->max_seqs * 4);
  w.pre_l = w.skip + cache_align((size_t)c->max_seqs * 4);
  w.pre_o = w.pre_l + cache_align((size_t)total_rows * heads * 4);
  w.ranges = w.pre_o + cache_align((size_t)total_rows * heads * c->dim * 4);
  w.range_tiles = total_rows * (heads / c->heads) / 256 + c->max_seqs + 1;
  w.total = w.ranges + cache_align((size_t)c->heads * w.range_tiles * 8);
  return w;
}

struct CommonParams {
  CacheDev c;
  int n, groups, G, sms;
  int64_t total_rows;
  const int32_t* seqs;
  const int64_t* row_off;
  const int32_t* group_off;
  int32_t* shared;
  int32_t* skip;
};

// One CTA a group: the leading table entries that all its sequences have in common, as far as every row of
// each sees those pages whole.
__global__ void __launch_bounds__(kThreads) common_kernel(CommonParams p) {
  __shared__ int sh_pages;
  pdl_wait();
  const CacheDev& c = p.c;
  const int g = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5;
  bool bad = t == 0 && (p.group_off[0] != 0 || p.group_off[p.groups] != p.n);
  for (int i = t; i < p.groups; i += kThreads) bad |= p.group_off[i + 1] < p.group_off[i];
  if (__syncthreads_or(bad)) {  // no groups, then
    for (int64_t i = g + (int64_t)t * p.groups; i < p.n; i += (int64_t)kThreads * p.groups) p.skip[i] = 0;
    if (t == 0) {
      p.shared[g] = 0;
      set_status(c.status, OCCAM_ERR_INVALID_ARG);
    }
    return;
  }
  const int a = p.group_off[g], b = p.group_off[g + 1];
  int pages = b - a < 2 ? 0 : c.max_pages;
  for (int i = a + t; i < b; i += kThreads) {
    const int s = p.seqs[i];
    const int64_t r0 = p.row_off[i], r1 = p.row_off[i + 1];
    const int len = (unsigned)s < (unsigned)c.max_seqs ? c.length[s] : -1;
    const bool fits = r0 >= 0 && r1 >= r0 && r1 <= p.total_rows && len >= r1 - r0 && len <= (int64_t)c.max_pages * c.T;
    pages = min(pages, fits ? (int)((len - (r1 - r0)) >> c.log2T) : 0);  // (what does not fit is recorded with the tails)
  }
  if (t == 0) sh_pages = c.max_pages;
  __syncthreads();
  atomicMin(&sh_pages, __reduce_min_sync(0xffffffffu, pages));
  __syncthreads();
  pages = sh_pages;
  if (pages > 0) {
    const int32_t* base = c.table + (int64_t)p.seqs[a] * c.max_pages;
    constexpr int COLS = 8;  // a lane's columns, all of them under way together
    for (int j0 = 0; j0 < pages; j0 += 32 * COLS) {
      int want[COLS];
#pragma unroll
      for (int k = 0; k < COLS; ++k) {
        const int j = j0 + k * 32 + lane;
        want[k] = j < pages && in_bounds(j < c.max_pages, c.status, kSiteAttendKey) ? base[j] : 0;
      }
      for (int i = a + 1 + warp; i < b; i += kThreads / 32) {
        const int32_t* row = c.table + (int64_t)p.seqs[i] * c.max_pages;
        int got[COLS];
#pragma unroll
        for (int k = 0; k < COLS; ++k) got[k] = j0 + k * 32 + lane < pages ? row[j0 + k * 32 + lane] : 0;
        int first = pages;
#pragma unroll
        for (int k = COLS - 1; k >= 0; --k)
          if (got[k] != want[k]) first = j0 + k * 32 + lane;
        first = __reduce_min_sync(0xffffffffu, first);
        if (lane == 0 && first < pages) atomicMin(&sh_pages, first);
      }
    }
    __syncthreads();
    pages = sh_pages;
  }
  // Whether it pays. In units of a row tile (256 query rows of a key head) against 128 keys on the tensor cores, 2 us of an
  // SM's time: a sequence of up to 32 such rows takes half of one, by the few-row kernel. (64 single tokens over 16 k
  // common tokens: 65 us shared, 480 not; three over 600: 35 and 21; 8 x 8 questions of 16 to 128 rows over 2,900, whose rows fill their
  // tiles without each other: 446 and 338.)
  float alone = 0.f;
  int64_t rows = 0;
  for (int i = a + t; i < b && pages > 0; i += kThreads) {
    const int m = (int)(p.row_off[i + 1] - p.row_off[i]);
    alone += row_tiles(m * p.G);
    rows += m;
  }
  for (int o = 16; o > 0; o >>= 1) {
    alone += __shfl_xor_sync(0xffffffffu, alone, o);
    rows += __shfl_xor_sync(0xffffffffu, rows, o);
  }
  __shared__ float sh_alone[kThreads / 32];
  __shared__ int64_t sh_rows[kThreads / 32];
  if (lane == 0) {
    sh_alone[warp] = alone;
    sh_rows[warp] = rows;
  }
  __syncthreads();
  alone = 0.f;
  rows = 0;
  for (int w = 0; w < kThreads / 32; ++w) {
    alone += sh_alone[w];
    rows += sh_rows[w];
  }
  const float all = (float)p.groups * c.heads;  // the other groups are taken to be alike
  const float saved = (alone - row_tiles((float)rows * p.G)) * (float)(pages << c.log2T) / 128.f * 2.f * all / p.sms;
  if (saved < kChain + (float)rows * p.G * all * kJoin) pages = 0;
  if (t == 0) p.shared[g] = pages << c.log2T;
  for (int i = a + t; i < b; i += kThreads) p.skip[i] = pages << c.log2T;
}

}  // namespace

#define OCCAM_TRY(x)                 \
  do {                               \
    int _rc = (x);                   \
    if (_rc != OCCAM_OK) return _rc; \
  } while (0)

extern "C" int occam_cache_shared_workspace_size(const occam_cache* cache, int64_t total_rows, int32_t heads, size_t* bytes) {
  OCCAM_TRY(check_cache(cache));
  if (!bytes || total_rows < 0 || total_rows > 0x7fffffff || heads < 1 || heads > 64 * cache->heads) return OCCAM_ERR_INVALID_ARG;
  *bytes = shared_ws(cache, total_rows, heads).total;
  return OCCAM_OK;
}

extern "C" int occam_cache_attend_shared(const occam_cache* cache, const occam_attend_args* a, const int32_t* group_off,
                                         int32_t n_groups, int32_t max_group_rows, void* workspace, size_t workspace_bytes,
                                         occam_stream_t stream) {
  const NvtxRange nvtx("occam_cache_attend_shared");
  launch_counter() = 0;
  OCCAM_TRY(check_cache(cache));
  if (a && a->keep) return OCCAM_ERR_UNSUPPORTED;
  CacheWs w;
  int rc = check_cache_ws(cache, 0, workspace, workspace_bytes, &w);
  SharedWs sw{};
  if (rc == OCCAM_OK && a && a->heads > 0 && a->total_rows > 0) {
    sw = shared_ws(cache, a->total_rows, a->heads);
    if (workspace_bytes < sw.total) rc = OCCAM_ERR_WORKSPACE;
  }
  AttendParams p{};
  OCCAM_TRY(attend_params(cache, a, workspace, rc, w, &p));
  if (n_groups < 0 || n_groups > cache->max_seqs || max_group_rows < 0 || (n_groups == 0) != (a->n == 0)) return OCCAM_ERR_INVALID_ARG;
  if (a->n == 0 || a->total_rows == 0) return OCCAM_OK;
  if (!group_off) return OCCAM_ERR_INVALID_ARG;
  p.group_off = group_off;
  int32_t* shared = ws_at<int32_t>(workspace, sw.shared);
  int32_t* skip = ws_at<int32_t>(workspace, sw.skip);
  p.shared = shared;
  p.skip = skip;
  p.pre_l = ws_at<float>(workspace, sw.pre_l);
  p.pre_o = ws_at<float>(workspace, sw.pre_o);
  p.ranges = ws_at<int2>(workspace, sw.ranges);
  p.range_tiles = sw.range_tiles;
  CommonParams m{p.c, a->n, n_groups, p.G, cache_sms(), a->total_rows, a->seqs, a->row_off, group_off, shared, skip};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (!launch_after(common_kernel, dim3((unsigned)n_groups), kThreads, 0, st, m)) return OCCAM_ERR_CUDA;
  AttendParams pre = p;
  pre.n = n_groups;
  pre.causal = 0;
  OCCAM_TRY(launch_attend<kPrefix>(pre, cache->dim, (int64_t)max_group_rows * p.G, n_groups == 1, st));
  return launch_attend<kTail>(p, cache->dim, (int64_t)a->max_rows * p.G, a->n == 1, st);
}
