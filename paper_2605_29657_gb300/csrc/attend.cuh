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
  int32_t* counters;  // per stretch: arrivals at an item that begins in it; at kAttendCtas: CTAs that have left
  float* part_o;
  float2* part_ml;
};

struct SeqInfo {
  int64_t row0;
  int rows, len, seq;
};

// Sequence i's rows and length; rows = 0 if it is not this launch's or if its offsets do
// not fit (recorded).
__device__ __forceinline__ SeqInfo attend_seq(const AttendParams& p, int i) {
  SeqInfo s;
  s.row0 = p.row_off[i];
  const int64_t r1 = p.row_off[i + 1];
  s.seq = p.seqs[i];
  s.rows = 0;
  s.len = 0;
  if ((unsigned)s.seq < (unsigned)p.c.max_seqs) {
    const int len = p.c.length[s.seq];
    if (s.row0 >= 0 && r1 >= s.row0 && r1 <= p.total_rows && len <= p.c.max_pages * p.c.T && r1 - s.row0 <= len) {
      s.len = len;
      const int64_t m = (r1 - s.row0) * p.G;
      if (m > p.row_lo && m <= p.row_hi) s.rows = (int)(r1 - s.row0);
      return s;
    }
  }
  set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
  return s;
}

__device__ __forceinline__ int div_group(const AttendParams& p, int x) {
  return (int)(((uint64_t)(uint32_t)x * p.g_mul) >> p.g_shift);
}

// Key tiles of KT keys that row tile rt (R rows) of a sequence can see, at least one.
template <int R, int KT>
__device__ __forceinline__ int key_tiles(const AttendParams& p, const SeqInfo& s, int rt) {
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
template <int R, int KT, int OVER>
__device__ __forceinline__ int64_t units_before(const AttendParams& p, const SeqInfo& s, int nrt) {
  if (!p.causal) return (int64_t)nrt * ((s.len + KT - 1) / KT + OVER);
  return (int64_t)nrt * OVER + floor_sum(nrt, (int64_t)p.G * KT, R, R - 1 + (int64_t)p.G * (s.len - s.rows + KT));
}
template <int R, int KT, int OVER>
__device__ __forceinline__ int64_t head_units(const AttendParams& p, const SeqInfo& s) {
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
template <int R, int KT, int OVER, int NT>
__device__ __forceinline__ LinePart attend_line(const AttendParams& p, int min_units, int64_t* sh, Line& l) {
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
template <int R, int KT, int OVER, int NT>
__device__ __forceinline__ void attend_find(const AttendParams& p, const Line& l, const LinePart& part, int c, int64_t* sh,
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
template <int R, int KT, int OVER, class W>
__device__ __forceinline__ bool walk_set(const AttendParams& p, const W& w, Walk& x, int in_item) {
  x.tiles = key_tiles<R, KT>(p, x.s, x.rt);
  x.ta = max(in_item - OVER, 0);
  x.tb = max(min((int)w.u1 - x.item - OVER, x.tiles), 0);
  return x.ta < x.tb;
}
// The next segment; false at the end of the stretch.
template <int R, int KT, int OVER, class W>
__device__ __forceinline__ bool walk_next(const AttendParams& p, const W& w, Walk& x) {
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
template <int R, int KT, int OVER, class W>
__device__ __forceinline__ bool walk_begin(const AttendParams& p, const W& w, Walk& x) {
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

}  // namespace occam
