// attend.cuh -- parameters and work partition shared by the attention kernels
// over the paged cache (internal header).
//
// The work is a line of units: for each sequence, key head and tile of query
// rows (token j, query head g of the key head's group: row j G + g) the key
// tiles that the tile's last row can see. Every CTA takes an equal stretch of
// the line. An item (sequence, head, row tile) that lies in one CTA's stretch
// is finished there; one that is split leaves a partial result (unnormalised
// sums, running maximum, sum) per CTA, and the CTA that arrives last adds them
// in order -- always the same order, so results do not depend on timing. An
// item's units are preceded by OVER empty ones: what beginning and ending an
// item costs, in key tiles, so that CTAs with many short items get fewer tiles.
// (Leaving 3/16 of the line in short stretches to the CTAs that are done first
// measured slower: 64 single tokens 100 us where equal stretches took 80 with the same kernel.)
#pragma once

#include "cache.cuh"

namespace occam {

struct AttendParams {
  CacheDev c;
  int layer, n, H, G, causal, bf16;
  int row_lo, row_hi;  // sequences with row_lo < rows * G <= row_hi are this launch's
  int64_t total_rows, q_row, total_keep;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  const int32_t* seqs;
  const int64_t* row_off;
  const uint8_t* keep;
  const int64_t* keep_off;
  float scale_log2;
  uint32_t g_mul, g_shift;  // x / G = x g_mul >> g_shift for 0 <= x < 2^31
  // attention over shared prefixes (see attend_shared.cu)
  const int32_t* group_off;  // prefixes: the sequences of each group
  const int32_t* shared;     // prefixes: tokens that a group's sequences have in common
  const int32_t* skip;       // tails: leading tokens of a sequence that its group's prefix stands for
  float* pre_o;              // results over the prefixes, normalised [total_rows, heads, dim]
  float* pre_l;              // and log2 sum_k 2^s_k
  int2* ranges;              // prefixes: the CTAs with parts of an item of the tensor-core kernel [key heads, range_tiles]
  int64_t range_tiles;
  int32_t* counters;  // per stretch: arrivals at an item that begins in it; at kAttendCtas: CTAs that have left
  float* part_o;
  float2* part_ml;
};

// What a launch attends over: the whole of each sequence; the prefix of a group of sequences, all their rows as
// one; or what is behind those prefixes, whose results are joined in.
enum { kWhole = 0, kPrefix = 1, kTail = 2 };
template <int MODE>
struct AttendCall : AttendParams {
  static constexpr int mode = MODE;
};

struct SeqInfo {
  int64_t row0;
  int rows, len, seq;
  int page0;  // (kTail) the first page's column
};
// The column of the first page
template <class P>
__device__ __forceinline__ int first_page(const P&, const SeqInfo& s) {
  return P::mode == kTail ? s.page0 : 0;
}

// Sequence i's rows and length; rows = 0 if it is not this launch's or if its offsets do
// not fit (recorded).
template <class P>
__device__ __forceinline__ SeqInfo attend_seq(const P& p, int i) {
  SeqInfo s;
  s.rows = 0;
  s.len = 0;
  s.page0 = 0;
  if constexpr (P::mode == kPrefix) {
    s.row0 = 0;
    s.seq = 0;
    const int len = p.shared[i];  // (0: nothing in common, or a group that does not fit)
    if (len <= 0) return s;
    const int a = p.group_off[i], b = p.group_off[i + 1];
    s.row0 = p.row_off[a];
    const int64_t r1 = p.row_off[b];
    s.seq = p.seqs[a];
    s.len = len;
    const int64_t m = (r1 - s.row0) * p.G;
    if (m > p.row_lo && m <= p.row_hi) s.rows = (int)(r1 - s.row0);
    return s;
  }
  s.row0 = p.row_off[i];
  const int64_t r1 = p.row_off[i + 1];
  s.seq = p.seqs[i];
  if ((unsigned)s.seq < (unsigned)p.c.max_seqs) {
    const int len = p.c.length[s.seq];
    if (s.row0 >= 0 && r1 >= s.row0 && r1 <= p.total_rows && len <= p.c.max_pages * p.c.T && r1 - s.row0 <= len) {
      s.len = len;
      const int64_t m = (r1 - s.row0) * p.G;
      if (m > p.row_lo && m <= p.row_hi) s.rows = (int)(r1 - s.row0);
      if constexpr (P::mode == kTail) {
        const int skip = p.skip[i];
        if (skip >= 0 && skip <= len - (r1 - s.row0) && (skip & (p.c.T - 1)) == 0) {
          s.page0 = skip >> p.c.log2T;
          s.len = len - skip;
          return s;
        }
        s.rows = 0;
      } else {
        return s;
      }
    }
  }
  set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
  return s;
}

__device__ __forceinline__ int div_group(const AttendParams& p, int x) {
  return (int)(((uint64_t)(uint32_t)x * p.g_mul) >> p.g_shift);
}

// Key tiles of KT keys that row tile rt (R rows) of a sequence can see, at least one.
template <int R, int KT, class P>
__device__ __forceinline__ int key_tiles(const P& p, const SeqInfo& s, int rt) {
  int keys = s.len;
  if (p.causal) keys = s.len - s.rows + div_group(p, min((rt + 1) * R - 1, s.rows * p.G - 1)) + 1;
  return (keys + KT - 1) / KT;
}
// sum of floor((a i + b) / m) over i = 0 .. n-1 (a, b >= 0): quotients are taken
// out, and the lattice points under the rest of the line are counted along
// the other axis
static __device__ __noinline__ int64_t floor_sum(int64_t n, int64_t m, int64_t a, int64_t b) {
  int64_t sum = 0;
  for (;;) {
    sum += (a / m) * (n * (n - 1) / 2) + (b / m) * n;
    a %= m;
    b %= m;
    const int64_t y = a * n + b;
    if (y < m) return sum;
    n = y / m;
    b = y % m;
    const int64_t t = m;
    m = a;
    a = t;
  }
}
// Units of the first nrt row tiles of a sequence's head. Row tile rt < the last sees
// base + 1 + floor(((rt + 1) R - 1) / G) keys.
template <int R, int KT, int OVER, class P>
__device__ __forceinline__ int64_t units_before(const P& p, const SeqInfo& s, int nrt) {
  if (!p.causal) return (int64_t)nrt * ((s.len + KT - 1) / KT + OVER);
  return (int64_t)nrt * OVER + floor_sum(nrt, (int64_t)p.G * KT, R, R - 1 + (int64_t)p.G * (s.len - s.rows + KT));
}
template <int R, int KT, int OVER, class P>
__device__ __forceinline__ int64_t head_units(const P& p, const SeqInfo& s) {
  if (s.rows == 0) return 0;
  const int nrt = (s.rows * p.G + R - 1) / R;
  return (nrt > 1 ? units_before<R, KT, OVER>(p, s, nrt - 1) : 0) + OVER + key_tiles<R, KT>(p, s, nrt - 1);
}

// Stretch c begins at c units / stretches. (Units are 31-bit numbers: 2^31 key
// tiles are hours of work.)
struct Line {
  int units, stretches;
  int q, r;  // units = q stretches + r
};
__device__ __forceinline__ int stretch_begin(const Line& l, int c) { return l.q * c + l.r * c / l.stretches; }
static __device__ __noinline__ int stretch_of(const Line& l, int u) {
  int c = min(max((int)((float)u * (float)l.stretches / (float)l.units), 0), l.stretches - 1);
  while (c + 1 < l.stretches && stretch_begin(l, c + 1) <= u) ++c;
  while (c > 0 && stretch_begin(l, c) > u) --c;
  return c;
}

// A stretch [u0, u1) and the item its first unit is in (in_item: u0's place in it).
struct Stretch {
  int u0, u1;
  int index, seq, head, row_tile, in_item;
};

// The line's length and this thread's part of it (its sequences i0 .. i1-1 begin at `at`).
struct LinePart {
  int at, mine;
  int i0, i1;
};
// Block-wide (NT threads, all of them); sh: NT / 32 + 4 int64 of shared memory.
// min_units: a stretch is no shorter.
template <int R, int KT, int OVER, int NT, class P>
__device__ __forceinline__ LinePart attend_line(const P& p, int min_units, int64_t* sh, Line& l) {
  constexpr int NWARP = NT / 32;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int per = (p.n + NT - 1) / NT;
  LinePart w;
  w.i0 = min(t * per, p.n);
  w.i1 = min(w.i0 + per, p.n);
  int64_t mine = 0;
  for (int i = w.i0; i < w.i1; ++i) mine += p.c.heads * head_units<R, KT, OVER>(p, attend_seq(p, i));
  int64_t incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 31) sh[warp] = incl;
  __syncthreads();
  int64_t before = 0, total = 0;
#pragma unroll
  for (int k = 0; k < NWARP; ++k) {
    if (k < warp) before += sh[k];
    total += sh[k];
  }
  if (total > 0x7fff0000) {
    set_status(p.c.status, OCCAM_ERR_UNSUPPORTED);
    total = 0;
  }
  w.at = (int)(before + incl - mine);
  w.mine = (int)mine;
  l.units = (int)total;
  l.stretches = min((int)gridDim.x, max(l.units / min_units, 1));
  l.q = l.units / l.stretches;
  l.r = l.units - l.q * l.stretches;
  return w;
}
// Stretch c, to all threads of the block.
template <int R, int KT, int OVER, int NT, class P>
__device__ __forceinline__ void attend_find(const P& p, const Line& l, const LinePart& part, int c, int64_t* sh,
                                            Stretch& w) {
  constexpr int NWARP = NT / 32;
  w.index = c;
  w.u0 = stretch_begin(l, c);
  w.u1 = stretch_begin(l, c + 1);
  int at = part.at;
  if (w.u0 >= at && w.u0 - at < part.mine) {
    for (int i = part.i0; i < part.i1; ++i) {
      const SeqInfo s = attend_seq(p, i);
      const int hu = (int)head_units<R, KT, OVER>(p, s);
      if (w.u0 < at + p.c.heads * hu) {
        const int off = w.u0 - at;
        const int h = off / hu, in_head = off - h * hu;
        int lo = 0, hi = (s.rows * p.G + R - 1) / R;  // the last row tile that begins at or before in_head
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (units_before<R, KT, OVER>(p, s, mid) <= in_head) lo = mid; else hi = mid;
        }
        sh[NWARP] = i;
        sh[NWARP + 1] = h;
        sh[NWARP + 2] = lo;
        sh[NWARP + 3] = in_head - (lo ? (int)units_before<R, KT, OVER>(p, s, lo) : 0);
        break;
      }
      at += p.c.heads * hu;
    }
  }
  __syncthreads();
  w.seq = (int)sh[NWARP];
  w.head = (int)sh[NWARP + 1];
  w.row_tile = (int)sh[NWARP + 2];
  w.in_item = (int)sh[NWARP + 3];
}

// The segment (an item's key tiles ta .. tb-1, those in the CTA's stretch) a role is at.
struct Walk {
  SeqInfo s;
  int item;  // the item's first unit
  int i, h, rt, tiles, ta, tb;
};
// False if no tile of the item lies in the stretch.
template <int R, int KT, int OVER, class P, class W>
__device__ __forceinline__ bool walk_set(const P& p, const W& w, Walk& x, int in_item) {
  x.tiles = key_tiles<R, KT>(p, x.s, x.rt);
  x.ta = max(in_item - OVER, 0);
  x.tb = max(min((int)w.u1 - x.item - OVER, x.tiles), 0);
  return x.ta < x.tb;
}
// The next segment; false at the end of the stretch.
template <int R, int KT, int OVER, class P, class W>
__device__ __forceinline__ bool walk_next(const P& p, const W& w, Walk& x) {
  x.item += OVER + x.tiles;
  if (x.item + OVER >= w.u1) return false;
  const int nrt = (x.s.rows * p.G + R - 1) / R;
  if (++x.rt == nrt) {
    x.rt = 0;
    if (++x.h == p.c.heads) {
      x.h = 0;
      do {
        x.s = attend_seq(p, ++x.i);
      } while (x.s.rows == 0);
    }
  }
  return walk_set<R, KT, OVER>(p, w, x, 0);
}
// The first segment; false if the stretch has none.
template <int R, int KT, int OVER, class P, class W>
__device__ __forceinline__ bool walk_begin(const P& p, const W& w, Walk& x) {
  x.i = w.seq;
  x.s = attend_seq(p, x.i);
  x.h = w.head;
  x.rt = w.row_tile;
  x.item = w.u0 - w.in_item;
  return walk_set<R, KT, OVER>(p, w, x, w.in_item) || walk_next<R, KT, OVER>(p, w, x);
}
// The first and the last stretch with tiles of the item.
template <int OVER>
__device__ __forceinline__ int2 item_stretches(const Line& l, const Walk& x) {
  return make_int2(stretch_of(l, x.item + OVER), stretch_of(l, x.item + OVER + x.tiles - 1));
}

// How a row's result over its tail, log2 sum l2, joins the one over the prefix (kTail, where there is one): a and b are
// the weights of the prefix's and the tail's normalised results, the return value is log2 of the whole sum.
__device__ __forceinline__ float join_prefix(const AttendParams& p, int64_t row, float l2, float& a, float& b) {
  const float pl = __ldcg(p.pre_l + row), m = fmaxf(pl, l2), base = m == -INFINITY ? 0.f : m;
  a = fast_exp2(pl - base);
  b = fast_exp2(l2 - base);
  const float sum = a + b, inv = sum == 0.f ? 0.f : 1.f / sum;
  a *= inv;
  b *= inv;
  return sum == 0.f ? -INFINITY : m + log2f(sum);
}

// Host side: checks a call's arguments and fills in the parameters. ws_rc: what the check of the workspace gave.
int attend_params(const occam_cache* cache, const occam_attend_args* a, void* workspace, int ws_rc, const CacheWs& w,
                  AttendParams* out);
// most: query rows a key head of one item's rows at most (it chooses the kernels); one: there is one such item.
template <int MODE>
int launch_attend(const AttendParams& p, int dim, int64_t most, bool one, cudaStream_t st);

}  // namespace occam
