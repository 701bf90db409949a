// attend_tc.cu -- attention over the paged 8-bit cache for many query rows per
// key head (questions, prefixes), on the fifth-generation tensor cores.
//
// The same running softmax as attend.cu, for 256 query rows (token, head of
// the group) against tiles of 128 keys. 4 D operations and one exponential a
// (row, key). A prefix of 8,257 tokens, 32 query and 8 key heads of 128 dims, takes 0.535 ms,
// 1.04 PFLOP/s: 3,800 cycles a tile where the products alone need 2,050 and shared
// memory's traffic (codes, their f16 form, operands: 384 KB) 3,070; bound by the
// round scores -> softmax -> P -> products, of which two halves a row tile are under way.
// (At 0.57 ms: without the softmax 0.47, without the exponentials 0.53, without the conversion 0.55.)
// One CTA an SM, 16 warps in five roles:
//  - warp 13 plans: it walks the key tiles, fills a ring of step records (masks,
//    scales, references) and has each page's block copied to shared memory as it is;
//    tiles without a seen key are left out, and a tile whose scales of v lie
//    more than 2^6 apart is taken 16 keys at a time;
//  - warps 8-11 turn the codes into f16 (exact) in the matrix layout
//    (128-byte swizzle), two stages deep;
//  - warps 12 and 14 issue the products: S = Q K^T into tensor memory, O += P V with P
//    read from tensor memory, each for a row tile of 128, 64 keys at a time: while a
//    row tile's softmax works on one half of its scores, the other half is multiplied
//    (128 keys at a time, 64 of P: measured slower, 0.61 ms where this took 0.55);
//  - warps 0-3 and 4-7 hold a row a thread: scores from tensor memory, maximum,
//    exponentials, P back over the scores as f16.
// O stays in tensor memory. It is rescaled only where a row's maximum grew by more than
// 2^8 since its last reference, or where v's scale left the window that P
// is held in; both references are undone at the end. P is rounded to f16 (see attend.cu), l sums the
// unrounded P.
#include <algorithm>
#include <atomic>

#include "attend.cuh"
#include "attend_tc.cuh"
#include "tc5.cuh"

using namespace occam;

namespace {

constexpr int kR = 256;        // query rows of an item
constexpr int kK = 128;        // keys of a tile
constexpr int kOver = 4;       // beginning and ending an item takes as long as this many tiles
constexpr int kGroup = 16;     // keys that share a page at least
constexpr int kThreads = 512;
constexpr int kRing = 4;
constexpr int kRegSoftmax = 168, kRegConvert = 88, kRegIssue = 88;  // 2 x 168 + 88 + 88 = 4 x 128
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr float kLazy = 8.f;             // log2 growth of a maximum before O is rescaled
constexpr float kLeast = 1.2e-38f;       // a score's factor: never 0, so that a hidden key's -inf stays
constexpr float kRhoKeep = 1.f / 64.f;
// P is held 2^7 times as large: at most 2^15 (f16 ends at 2^16), and what is 2^-21 of a row's
// reference still has f16's 11 bits; below 2^-32 it is lost. l stays in true units, O's factor is taken
// back by the last reference.
constexpr float kLift = 7.f, kUnlift = 1.f / 128.f;
constexpr float kRhoSpan = 8.6736174e-19f;  // 2^-60

struct Step {
  int tile;
  int open;           // every row of the item sees the whole tile
  uint32_t zero;      // bit g: v's scale is 0 in group g
  int end;            // 1: no more steps of this segment (an item, or the CTA's part of one); 2: nor segments
  int row_tiles;      // 1 or 2
  uint32_t seen[4];   // bit k: key k of the tile may be seen
  float ks[8];        // scale of k, per 16 keys
  float lr[8];        // log2(scale of v / rho) + kLift
  float rr[8];        // kUnlift rho / scale of v
  float fall;         // O's factor: rho before / rho now
  float rho;          // kUnlift rho
};

struct Shared {
  uint64_t q_full[2], k_full[2], k_free[2], v_full[2], v_free[2], s_full[2][2], p_full[2][2], o_done[2][2], step_full[kRing],
      step_free[kRing], raw_full[2], raw_free[2], meet, drain;
  Step step[kRing];
  Line line;
  int u0, u1;   // the CTA's stretch (see Stretch)
  int seq, head, row_tile, in_item;
  uint32_t tmem;
  int stop;            // a wait ran out
  int last;
  int left;            // the last CTA to leave
  int any_nan[4];
  alignas(16) int nan_first[4][128];  // (first the scratch of attend_line: 8-byte words)
};
constexpr int kSharedBytes = 3072;
static_assert(sizeof(Shared) <= kSharedBytes, "7 tiles of 32 KB and this are all of an SM's shared memory");

__device__ __forceinline__ uint64_t desc_kmajor(uint32_t saddr) { return tc::sdesc_sw128(saddr); }
// rows of the summed index, 64 columns (128 bytes) a block, blocks 16 KB apart
__device__ __forceinline__ uint64_t desc_mnmajor(uint32_t saddr) { return tc::sdesc_mn_sw128(saddr, 16384); }
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool trans_b) { return tc::idesc16(false, M, N, trans_b); }
using tc::add2;
using tc::elect_one;
using tc::fma2;
using tc::mma_ts;
using tc::pack_f16;
using tc::tmem_ld16;
using tc::tmem_st16;
using tc::wait_ld;

// (prefixes) an item's place among its head's
__device__ __forceinline__ int range_at(const AttendParams& p, int64_t row0, int i, int rt) { return (int)(row0 * p.G / kR) + i + rt; }
__device__ __forceinline__ int range_at(const AttendParams& p, const Walk& x) { return range_at(p, x.s.row0, x.i, x.rt); }
__device__ __forceinline__ int row_tiles(const AttendParams& p, const Walk& x) {
  return x.s.rows * p.G - x.rt * kR > 128 ? 2 : 1;
}

// ---------------------------------------------------------------- planning
__device__ __forceinline__ uint32_t pick(const uint32_t (&v)[4], int k) {
  const uint32_t lo = k & 1 ? v[1] : v[0], hi = k & 1 ? v[3] : v[2];
  return k & 2 ? hi : lo;
}

// What the planning warp knows of a key tile; lane l holds the page and scales of group l & 7 (16 keys).
struct Tile {
  int tile, page;
  float ks, vs;
  uint32_t seen[4];
};

// (One warp runs this once a step, so its latency is the step's: reductions are votes and
// integer redux, masks without flags are arithmetic, divisions are left out where all scales agree.)
struct Plan {
  const AttendParams& p;
  const Walk& x;
  const int lane;
  const int32_t* table;
  const uint8_t* flags;
  const float* ks0;  // scales of page 0 in this layer and head
  const float* vs0;
  int n_flags;
  int column;  // of the item's first page

  __device__ Plan(const AttendParams& p_, const Walk& x_, int lane_) : p(p_), x(x_), lane(lane_) {}

  __device__ __forceinline__ void item(int first_column) {
    column = first_column;
    table = p.c.table + (int64_t)x.s.seq * p.c.max_pages + column;
    const int64_t b = (int64_t)p.layer * p.c.pages * p.c.heads + x.h;
    ks0 = p.c.k_scale + b;
    vs0 = p.c.v_scale + b;
    flags = nullptr;
    n_flags = 0;
    if (p.keep) {
      const int64_t k0 = p.keep_off[x.i], k1 = p.keep_off[x.i + 1];
      if (k0 >= 0 && k1 >= k0 && k1 <= p.total_keep) {
        flags = p.keep + k0;
        n_flags = (int)min(k1 - k0, (int64_t)x.s.len);
      } else {
        set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
      }
    }
  }
  // page and raw flags (loads in flight)
  __device__ __forceinline__ void look(Tile& t, int tile) const {
    t.tile = tile;
    const int first = tile * kK + (lane & 7) * kGroup;
    t.page = 0;
    if (first < x.s.len && in_bounds(column + (first >> p.c.log2T) < p.c.max_pages, p.c.status, kSiteAttendKey))
      t.page = table[first >> p.c.log2T];
    if (tile * kK < n_flags) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int key = tile * kK + 32 * k + lane;
        const bool flag = key < n_flags && in_bounds(flags + key < p.keep + p.total_keep, p.c.status, kSiteAttendKey);
        t.seen[k] = flag ? flags[key] : 1u;
      }
    }
  }
  // masks, and the scales (loads in flight)
  __device__ __forceinline__ void settle(Tile& t) const {
    const bool bad = (unsigned)t.page >= (unsigned)p.c.pages;
    const int keys = x.s.len - t.tile * kK;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int n = keys - 32 * k;
      uint32_t see = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
      if (t.tile * kK < n_flags) see &= __ballot_sync(0xffffffffu, t.seen[k] != 0);
      t.seen[k] = see;
    }
    const unsigned wrong = __ballot_sync(0xffffffffu, bad) & 0xff;
    if (wrong) {
      set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
      if (bad) t.page = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if ((wrong >> (2 * k)) & 1) t.seen[k] &= 0xffff0000u;
        if ((wrong >> (2 * k + 1)) & 1) t.seen[k] &= 0x0000ffffu;
      }
    }
    t.ks = ks0[(int64_t)t.page * p.c.heads];
    t.vs = vs0[(int64_t)t.page * p.c.heads];
  }
  // groups with a seen key, a bit each
  __device__ __forceinline__ uint32_t groups(const Tile& t) const {
    const bool h = (pick(t.seen, (lane & 7) >> 1) >> (16 * (lane & 1))) & 0xffffu;
    return __ballot_sync(0xffffffffu, h) & 0xff;
  }
  // the largest and least positive, finite scale of v in those groups (positive floats order as integers)
  __device__ __forceinline__ void range(const Tile& t, uint32_t with, float& hi, float& lo) const {
    const bool h = ((with >> (lane & 7)) & 1) && t.vs > 0.f && t.vs <= 3.4e38f;
    hi = __uint_as_float(__reduce_max_sync(0xffffffffu, h ? __float_as_uint(t.vs) : 0u));
    lo = __uint_as_float(__reduce_min_sync(0xffffffffu, h ? __float_as_uint(t.vs) : 0x7f800000u));
  }
};

// ---------------------------------------------------------------- conversion
// A pass of the four warps takes RPP key rows, LPR lanes a row, 16 codes a lane. Row r of every
// pass has the same r & 7, so a lane's swizzled places are the same in each.
template <int D>
struct Convert {
  static constexpr int LPR = D / 16;
  static constexpr int RPP = 128 / LPR;  // 16 (D = 128) or 32 rows
  static constexpr int PASSES = 128 / RPP;

  const int row0, c;   // row of pass 0, piece of the row
  int place0, place1;  // this lane's two 16-byte pieces in a matrix, pass 0
  uint32_t swap;       // all ones: the odd piece is written first

  __device__ Convert(int lane, int warp) : row0(warp * (32 / LPR) + lane / LPR), c(lane % LPR) {
    // [D / 64][128 keys][64 dims], 128-byte swizzle. The two halves of a row start at the same
    // bank: their lanes write their even and odd pieces in opposite order.
    const int odd = c >> 2;
    swap = 0u - (uint32_t)odd;
    const int base = odd * 16384 + row0 * 128, idx = 2 * (c & 3);
    place0 = base + (((idx + odd) ^ (row0 & 7)) << 4);
    place1 = base + (((idx + 1 - odd) ^ (row0 & 7)) << 4);
  }
  __device__ __forceinline__ void read(uint4 (&r)[PASSES], const unsigned char* raw) const {
    const uint4* at = reinterpret_cast<const uint4*>(raw + row0 * D + c * 16);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) r[i] = at[i * RPP * D / 16];
  }
  // Returns once the values are in registers: an arrival does not wait for loads under way, and the copy that it lets
  // begin can overtake them where products take most of the shared memory's reads. (What it sleeps for changes nothing;
  // a fence in its place did not wait for them either.)
  __device__ __forceinline__ void landed(const uint4 (&r)[PASSES]) const {
    uint32_t all = 0;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) all |= r[i].x | r[i].y | r[i].z | r[i].w;
    if (all == 0x80000001u) __nanosleep(1);
  }
  // hidden rows may be anything: zeros
  __device__ __forceinline__ void mask(uint4 (&r)[PASSES], const uint32_t* seen) const {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const uint32_t m = 0u - ((seen[i * RPP / 32] >> (row0 + i * RPP % 32)) & 1u);
      r[i] = make_uint4(r[i].x & m, r[i].y & m, r[i].z & m, r[i].w & m);
    }
  }
  __device__ __forceinline__ void store(const uint4 (&r)[PASSES], unsigned char* base) const {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const uint32_t w0 = (r[i].x & ~swap) | (r[i].z & swap), w1 = (r[i].y & ~swap) | (r[i].w & swap);
      const uint32_t w2 = (r[i].z & ~swap) | (r[i].x & swap), w3 = (r[i].w & ~swap) | (r[i].y & swap);
      *reinterpret_cast<uint4*>(base + place0 + i * (RPP * 128)) =
          make_uint4(e4m3x2_f16x2(w0), e4m3x2_f16x2_hi(w0), e4m3x2_f16x2(w1), e4m3x2_f16x2_hi(w1));
      *reinterpret_cast<uint4*>(base + place1 + i * (RPP * 128)) =
          make_uint4(e4m3x2_f16x2(w2), e4m3x2_f16x2_hi(w2), e4m3x2_f16x2(w3), e4m3x2_f16x2_hi(w3));
    }
  }
  __device__ __forceinline__ bool nans(const uint4 (&r)[PASSES]) const {
    uint32_t hit = 0;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const uint32_t w[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) hit |= (w[k] & 0x7f7f7f7fu) + 0x01010101u;
    }
    return (hit & 0x80808080u) != 0;
  }
  // The rare cases work on the matrix, on this lane's own pieces, in rolled loops.
  // Values of scale 0 are 0.
  __device__ __forceinline__ void clear(uint32_t zero, unsigned char* base) const {
#pragma unroll 1
    for (int i = 0; i < PASSES; ++i) {
      if ((zero >> ((row0 + i * RPP) / kGroup)) & 1) {
        *reinterpret_cast<uint4*>(base + place0 + i * (RPP * 128)) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(base + place1 + i * (RPP * 128)) = make_uint4(0, 0, 0, 0);
      }
    }
  }
  // NaN values that some row does not see are taken out and the token noted.
  __device__ __forceinline__ void note(int tile, unsigned char* base, int* first, int* any) const {
    *any = 1;
#pragma unroll 1
    for (int i = 0; i < PASSES; ++i) {
#pragma unroll 1
      for (int b = 0; b < 16; ++b) {
        uint16_t* v = reinterpret_cast<uint16_t*>(base + ((b >> 3) != (int)(swap & 1) ? place1 : place0) + i * (RPP * 128)) + (b & 7);
        if ((*v & 0x7fff) > 0x7c00) {
          atomicMin(&first[c * 16 + b], tile * kK + row0 + i * RPP);
          *v = 0;
        }
      }
    }
  }
};

// the block of codes of one page and head
__device__ __forceinline__ void tma_block(void* dst, const CUtensorMap* map, int row, int page, uint64_t* bar) {
  tc::tma_load_3d(dst, map, 0, row, page, bar);
}

// a bounded wait on a barrier phase; false (recorded) if it ran out or another role gave up
__device__ __forceinline__ bool wait_long(uint64_t* bar, uint32_t parity, volatile int* stop, int32_t* status) {
  const uint64_t t0 = tc::globaltimer();
  while (!tc::bar_try(bar, parity)) {
    if (*stop || tc::globaltimer() - t0 > kWaitNs) {
      *stop = 1;
      set_status(status, OCCAM_ERR_TIMEOUT);
      return false;
    }
  }
  return true;
}
#define TC_WAIT(bar, parity)                                                                               \
  if (!tc::bar_try(&(bar), (parity)) && !wait_long(&(bar), (parity), &sh.stop, p.c.status)) return;
// the 256 softmax threads meet
#define TC_MEET()                        \
  do {                                   \
    tc::bar_arrive(&sh.meet);            \
    TC_WAIT(sh.meet, met & 1)            \
    ++met;                               \
  } while (0)

template <int D, class P>
__device__ __forceinline__ void plan_role(const P& p, Shared& sh, const CUtensorMap& map_k, const CUtensorMap& map_v,
                                          unsigned char* raw) {
  const int lane = threadIdx.x & 31;
  Walk x;
  if (!walk_begin<kR, kK, kOver>(p, sh, x)) return;
  Plan f(p, x, lane);
  uint32_t n = 0, j = 0;  // step records, steps so far
  uint32_t seg = 0;
  for (bool again = true; again; ++seg) {
    f.item(first_page(p, x.s));
    // The notes of four segments ago: a segment has two records at least, so every row tile has given back that one's last.
    if (sh.any_nan[seg & 3]) {
      for (int d = lane; d < D; d += 32) sh.nan_first[seg & 3][d] = 0x7fffffff;
      __syncwarp();
      if (lane == 0) sh.any_nan[seg & 3] = 0;
      __syncwarp();
    }
    const int common = p.causal ? x.s.len - x.s.rows + div_group(p, x.rt * kR) + 1 : x.s.len;
    const int end = x.tb - 1, tiles2 = row_tiles(p, x);
    float rho = 0.f, rho_max = 0.f;
    // tiles in the order of their stages: in hand (cur), masks and scales (nxt), page and flags (far)
    Tile cur, nxt, far;
    int groups = 0;     // groups of the present tile still to be taken one by one
    uint32_t whole[4];  // the present tile's mask, while it is taken so
    cur.tile = x.ta - 3;  // (two turns of the stages bring the first tile to nxt)
    cur.seen[0] = cur.seen[1] = cur.seen[2] = cur.seen[3] = 0;
    nxt = far = cur;
    nxt.tile = x.ta - 2;
    far.tile = x.ta - 1;
    far.page = 0;
    for (bool none = true;; none = false) {
      // the next step (tiles without a seen key are passed over)
      int only = -1;  // the group that is taken alone
      if (groups) {
        only = __ffs(groups) - 1;
        groups &= groups - 1;
      } else {
        bool found = false;
#pragma unroll 1
        while (!found && cur.tile < end) {
          cur = nxt;
          nxt = far;
          f.settle(nxt);
          f.look(far, min(nxt.tile + 1, end));
          found = cur.tile >= x.ta && (cur.seen[0] | cur.seen[1] | cur.seen[2] | cur.seen[3]) != 0;
        }
        if (!found && !none) break;  // (where nothing is seen, one step of hidden keys gives the rows their zeros)
      }
      uint32_t with = only >= 0 ? 1u << only : f.groups(cur);
      float hi, lo;
      f.range(cur, with, hi, lo);
      if (only < 0 && lo < hi * kRhoKeep) {
        // scales of v too far apart for one reference: the groups with a seen key one by one
        only = __ffs(with) - 1;
        groups = with & (with - 1);
        with = 1u << only;
        f.range(cur, with, hi, lo);
#pragma unroll
        for (int k = 0; k < 4; ++k) whole[k] = cur.seen[k];
      }
      if (only >= 0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) cur.seen[k] = (only >> 1) == k ? whole[k] & (0xffffu << (16 * (only & 1))) : 0u;
      }
      // v's reference, and O's factor
      float fall = 1.f;
      if (hi > rho || lo < rho * kRhoKeep) {
        const float to = hi > rho ? hi : fmaxf(hi, rho_max * kRhoSpan);
        fall = rho / to;
        rho = to;
        rho_max = fmaxf(rho_max, to);
      }
      // hidden groups take no part; a scale of 0 makes values of 0
      const bool has = (with >> (lane & 7)) & 1, real = has && cur.vs != 0.f;
      const uint32_t zero = with & ~__ballot_sync(0xffffffffu, real);
      float lr = 0.f, rr = 1.f;
      if (__any_sync(0xffffffffu, real && cur.vs != rho)) {
        if (real && cur.vs != rho) {
          lr = log2f(cur.vs / rho);
          rr = rho / cur.vs;
        }
      }
      TC_WAIT(sh.step_free[n % kRing], ((n / kRing) & 1) ^ 1);
      Step& s = sh.step[n % kRing];
      if (lane < 8) {
        s.ks[lane] = has ? cur.ks : 1.f;
        s.lr[lane] = lr + kLift;
        s.rr[lane] = rr * kUnlift;
      }
      if (lane == 8) {
#pragma unroll
        for (int k = 0; k < 4; ++k) s.seen[k] = cur.seen[k];
        s.zero = zero;
      }
      if (lane == 0) {
        s.tile = cur.tile;
        s.open = (cur.seen[0] & cur.seen[1] & cur.seen[2] & cur.seen[3]) == 0xffffffffu && (cur.tile + 1) * kK <= common;
        s.end = 0;
        s.row_tiles = tiles2;
        s.fall = fall;
      }
      __syncwarp();
      if (lane == 0) tc::bar_arrive(&sh.step_full[n % kRing]);
      ++n;
      // the blocks of the pages with a seen key: lane b takes the tile's b-th page, 1 << log_gp groups each
      const int T = p.c.T, log_gp = p.c.log2T - 4;
      const int page = __shfl_sync(0xffffffffu, cur.page, (lane << log_gp) & 7);
      const bool want = lane < (8 >> log_gp) && ((with >> (lane << log_gp)) & ((1u << (1 << log_gp)) - 1u)) != 0;
      const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, want)) * T * D;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        TC_WAIT(sh.raw_free[kv], (j & 1) ^ 1);
        if (lane == 0) tc::bar_expect_tx(&sh.raw_full[kv], bytes);
        __syncwarp();
        if (want)
          tma_block(raw + kv * (kK * D) + lane * T * D, kv ? &map_v : &map_k, x.h * T, p.layer * p.c.pages + page,
                    &sh.raw_full[kv]);
      }
      ++j;
    }
    // the end of the segment
    TC_WAIT(sh.step_free[n % kRing], ((n / kRing) & 1) ^ 1);
    again = walk_next<kR, kK, kOver>(p, sh, x);
    if (lane == 0) {
      sh.step[n % kRing].end = again ? 1 : 2;
      sh.step[n % kRing].rho = rho * kUnlift;
      tc::bar_arrive(&sh.step_full[n % kRing]);
    }
    ++n;
  }
}

template <int D>
__device__ __forceinline__ void convert_role(const AttendParams& p, Shared& sh, unsigned char* k_smem, unsigned char* v_smem,
                                             const unsigned char* raw) {
  constexpr int kBytes = kK * D * 2;
  const int lane = threadIdx.x & 31;
  const Convert<D> f(lane, (threadIdx.x >> 5) & 3);
  uint32_t j = 0, seg = 0;
#pragma unroll 1
  for (uint32_t n = 0;; ++n) {
    TC_WAIT(sh.step_full[n % kRing], (n / kRing) & 1);
    const Step& s = sh.step[n % kRing];
    const int end = s.end;
    if (!end) {
      const bool full = (s.seen[0] & s.seen[1] & s.seen[2] & s.seen[3]) == 0xffffffffu;
      const int st = j & 1;
#pragma unroll 1
      for (int kv = 0; kv < 2; ++kv) {
        uint4 r[Convert<D>::PASSES];
        TC_WAIT(sh.raw_full[kv], j & 1);
        f.read(r, raw + kv * (kK * D));
        f.landed(r);
        if (!full) f.mask(r, s.seen);
        __syncwarp();
        if (lane == 0) tc::bar_arrive(&sh.raw_free[kv]);
        unsigned char* to = (kv ? v_smem : k_smem) + st * kBytes;
        TC_WAIT(*(kv ? &sh.v_free[st] : &sh.k_free[st]), ((j >> 1) & 1) ^ 1);
        f.store(r, to);
        if (kv) {
          if (!s.open && f.nans(r)) f.note(s.tile, to, sh.nan_first[seg & 3], &sh.any_nan[seg & 3]);
          if (s.zero) f.clear(s.zero, to);
        }
        tc::fence_proxy_async();
        tc::bar_arrive(kv ? &sh.v_full[st] : &sh.k_full[st]);
      }
      ++j;
    } else {
      ++seg;
    }
    __syncwarp();
    if (lane == 0) tc::bar_arrive(&sh.step_free[n % kRing]);
    if (end == 2) return;
  }
}

// ---------------------------------------------------------------- issuing
// One warp for each row tile t. The whole warp walks through the steps (so that
// branches are the same for every lane); one elected lane issues. (A single
// warp for both was the slowest part: about 70 cycles an instruction.)
template <int D>
__device__ __forceinline__ void mma_role(const AttendParams& p, Shared& sh, uint32_t q_smem, uint32_t k_smem,
                                         uint32_t v_smem, uint32_t tmem, int t) {
  constexpr int kBytes = kK * D * 2;
  constexpr uint32_t id_s = idesc_f16(128, 64, false), id_o = idesc_f16(128, D, true);
  const uint64_t dq = desc_kmajor(q_smem + t * kBytes), dk = desc_kmajor(k_smem), dv = desc_mnmajor(v_smem);
  uint32_t n = 0, j = 0, it = 0;  // step records, steps, steps of this row tile
  int end = 0;
  uint32_t queries = 0;  // segments of this row tile
  while (end != 2) {
    bool mine = true;
    end = 0;
    // Pass k: by halves h, O += P V of step k - 1, then S of step k in the place of that P.
    // (Rolled: the roles together have to stay within the instruction cache.
    // A descriptor's address field counts 16 bytes.)
#pragma unroll 1
    for (uint32_t k = 0; !end; ++k) {
#pragma unroll 1
      for (uint32_t h = 0; h < 2; ++h) {
        if (k > 0) {
          if (h == 0) TC_WAIT(sh.v_full[(j - 1) & 1], ((j - 1) >> 1) & 1);
          if (mine) {
            TC_WAIT(sh.p_full[t][h], it & 1);
            tc::fence_after();
            if (elect_one()) {
              const uint64_t vd = dv + ((j - 1) & 1) * (kBytes >> 4) + h * (64 * 128 >> 4);
              const uint32_t o_at = tmem + 256 + t * 128, p_at = tmem + t * 128 + h * 64;
#pragma unroll
              for (int q = 0; q < 4; ++q)
                mma_ts(o_at, p_at + q * 8, vd + q * (2048 >> 4), id_o, q > 0 ? 1u : (k > 1 || h > 0 ? 1u : 0u));
              tc::mma_commit(&sh.o_done[t][h]);
            }
            __syncwarp();
          }
        }
        if (h == 0) {
          TC_WAIT(sh.step_full[n % kRing], (n / kRing) & 1);
          end = sh.step[n % kRing].end;
          if (!end) {
            mine = t < sh.step[n % kRing].row_tiles;
            if (k == 0 && mine) {
              TC_WAIT(sh.q_full[t], queries & 1);
              ++queries;
            }
            TC_WAIT(sh.k_full[j & 1], (j >> 1) & 1);
            tc::fence_after();
          }
        }
        if (!end && mine) {
          if (elect_one()) {
            const uint64_t kd = dk + (j & 1) * (kBytes >> 4) + h * (64 * 128 >> 4);
            const uint32_t s_at = tmem + t * 128 + h * 64;
#pragma unroll
            for (int q = 0; q < D / 16; ++q) {
              const int o = (q >> 2) * (16384 >> 4) + (q & 3) * 2;
              tc::mma_bf16(s_at, dq + o, kd + o, id_s, q > 0);
            }
            tc::mma_commit(&sh.s_full[t][h]);
          }
          __syncwarp();
        }
      }
      if (k > 0 && mine) ++it;
      // (without products of its own the warp just arrives: it has waited for the same stages)
      if (elect_one()) {
        if (k > 0) mine ? tc::mma_commit(&sh.v_free[(j - 1) & 1]) : tc::bar_arrive(&sh.v_free[(j - 1) & 1]);
        if (!end) mine ? tc::mma_commit(&sh.k_free[j & 1]) : tc::bar_arrive(&sh.k_free[j & 1]);
        tc::bar_arrive(&sh.step_free[n % kRing]);
      }
      __syncwarp();
      ++n;
      if (!end) ++j;
    }
  }
}

// ---------------------------------------------------------------- a row a thread
// The warp's 32 query rows (from row `first` of the item's tile) as f16 in the
// matrix layout, each scaled by a power of two of its own; lane l gets row l's scale
// (with the softmax's). D / 8 lanes take a row; the copies are all in flight at
// once, and each lane converts in place what it copied.
template <int D, bool BF16>
__device__ __forceinline__ float load_queries(const AttendParams& p, const Walk& x, int first, unsigned char* q_smem, int lane) {
  constexpr int LPR = D / 8, RPI = 32 / LPR, N = 32 / RPI;
  const int c = lane % LPR, sub = lane / LPR, rows = x.s.rows * p.G;
  unsigned char* mine = q_smem + (c >> 3) * 16384;
  auto piece = [&](int i) {
    const int r = (first & 127) + i * RPI + sub;
    return mine + r * 128 + (((c & 7) ^ (r & 7)) << 4);
  };
  const uint16_t* row_at = nullptr;  // lane l's row
  {
    const int at = x.rt * kR + first + lane, tok = div_group(p, at);
    if (at < rows && in_bounds(x.s.row0 + tok < p.total_rows && x.h * p.G + at - tok * p.G < p.H, p.c.status, kSiteAttendRow))
      row_at = p.q + (x.s.row0 + tok) * p.q_row + (int64_t)(x.h * p.G + at - tok * p.G) * D;
  }
#pragma unroll 4
  for (int i = 0; i < N; ++i) {
    const uint64_t from = __shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(row_at), i * RPI + sub);
    tc::cp_async16(piece(i), from ? reinterpret_cast<const uint16_t*>(from) + c * 8 : p.q, from ? 16 : 0);
  }
  cp_async_commit();
  cp_async_wait<0>();
  // The largest magnitude of each row (magnitudes order as integers; a NaN does not matter, its
  // row is NaN): this lane's share of the N = LPR rows, then exchanges that halve the rows a lane
  // has and double the lanes it has seen, until lane c has row c's (of its `sub`).
  static_assert(N == LPR, "");
  uint32_t top[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint4 v = *reinterpret_cast<const uint4*>(piece(i));
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    top[i] = max(m & 0xffffu, m >> 16);
  }
#pragma unroll
  for (int n = N / 2; n > 0; n >>= 1) {
    const bool high = c & n;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const uint32_t give = high ? top[i] : top[i + n], keep = high ? top[i + n] : top[i];
      top[i] = max(keep, __shfl_xor_sync(0xffffffffu, give, n));
    }
  }
  // a row's power of two: largest value in [2^14, 2^15), as in attend.cu
  const float amax = BF16 ? __uint_as_float(top[0] << 16) : __half2float(__ushort_as_half((unsigned short)top[0]));
  const int e = amax == 0.f ? 0 : max((__float_as_int(amax) >> 23) - 127 - 14, -112);
#pragma unroll 4
  for (int i = 0; i < N; ++i) {
    uint4* at = reinterpret_cast<uint4*>(piece(i));
    const uint4 v = *at;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const float up = __int_as_float((127 - __shfl_sync(0xffffffffu, e, sub * LPR + i)) << 23);
    uint32_t r[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 f = BF16 ? make_float2(bf16_lo(w[k]), bf16_hi(w[k])) : __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
      r[k] = pack_f16(f.x * up, f.y * up);
    }
    *at = make_uint4(r[0], r[1], r[2], r[3]);
  }
  // lane l's own row is row l % RPI of the loop's l / RPI-th
  const float scale = __int_as_float((127 + __shfl_sync(0xffffffffu, e, (lane % RPI) * LPR + lane / RPI)) << 23);
  return scale * p.scale_log2;
}

template <bool BF16>
__device__ __forceinline__ uint32_t out_pair(float a, float b) {
  if (BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  return pack_f16(a, b);
}

template <int D, bool BF16, class P>
__device__ __forceinline__ void softmax_role(const P& p, Shared& sh, unsigned char* q_smem,
                                             uint32_t tmem, int t) {
  const int r = threadIdx.x & 127, lane = threadIdx.x & 31;
  const uint32_t lanes = (uint32_t)(r & ~31) << 16;
  const uint32_t s_at = tmem + t * 128 + lanes, o_at = tmem + 256 + t * 128 + lanes;
  Walk x;
  if (!walk_begin<kR, kK, kOver>(p, sh, x)) return;
  uint32_t n = 0, it = 0, seg = 0, met = 0;
  do {
    const bool mine = t < row_tiles(p, x);
    const int row = t * 128 + r, at = x.rt * kR + row;
    const bool there = at < x.s.rows * p.G;
    float qscale = 0.f;
    if (mine) qscale = load_queries<D, BF16>(p, x, row & ~31, q_smem + t * kK * D * 2, lane);
    tc::fence_proxy_async();
    // (a barrier a row tile: the warps of one that has no rows in these segments are ahead of the other's)
    if (mine) tc::bar_arrive(&sh.q_full[t]);
    const int limit = !there ? 0 : p.causal ? x.s.len - x.s.rows + div_group(p, at) + 1 : x.s.len;  // keys this row sees
    const int common = p.causal ? x.s.len - x.s.rows + div_group(p, x.rt * kR + t * 128) + 1 : x.s.len;
    float ref = -INFINITY, top = -INFINITY, l = 0.f, rho = 0.f;
    for (bool begin = true;; begin = false) {
      TC_WAIT(sh.step_full[n % kRing], (n / kRing) & 1);
      const Step& st = sh.step[n % kRing];
      const bool end = st.end != 0;
      if (end) rho = st.rho;
      if (!end && mine) {
        const int tile = st.tile;
        const bool open = (st.seen[0] & st.seen[1] & st.seen[2] & st.seen[3]) == 0xffffffffu && (tile + 1) * kK <= common;
#pragma unroll 1
        for (int h = 0; h < 2; ++h, ++it) {
          TC_WAIT(sh.s_full[t][h], (it >> 1) & 1);
          tc::fence_after();
          // The row's scores of 64 keys: the maximum, and hidden ones -inf. The exponentials read them
          // again, 32 at a time in a rolled loop: 64 held in registers took 0.63 ms where this took 0.61
          // (32 questions with keep flags), a rolled loop here too 0.63.
          float m = top;
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t v[32];
            tc::tmem_ld32(s_at + 64 * h + 32 * q, v);
            wait_ld(v);
            if (!open) {
              const int lim = limit - tile * kK - 64 * h - 32 * q;
              const uint32_t see = st.seen[2 * h + q] & (lim >= 32 ? 0xffffffffu : lim <= 0 ? 0u : (1u << lim) - 1u);
#pragma unroll
              for (int k = 0; k < 32; ++k) v[k] = (see >> k) & 1 ? v[k] : 0xff800000u;
              tc::tmem_st32(s_at + 64 * h + 32 * q, v);
            }
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              const float f = fmaxf(st.ks[4 * h + 2 * q + g] * qscale, kLeast);
              float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
              for (int k = 0; k < 8; k += 2) {
                x0 = tc::fmax3(x0, __uint_as_float(v[16 * g + k]), __uint_as_float(v[16 * g + k + 1]));
                x1 = tc::fmax3(x1, __uint_as_float(v[16 * g + 8 + k]), __uint_as_float(v[16 * g + 9 + k]));
              }
              m = fmaxf(m, fmaxf(x0, x1) * f);
            }
          }
          if (!open) tc::tmem_wait_st();
          top = m;
          float fall = h == 0 ? st.fall : 1.f;
          bool move = fall != 1.f;
          if (m > ref + kLazy || ref == -INFINITY) {
            if (m != ref) {
              const float by = ref == -INFINITY ? 0.f : fast_exp2(ref - m);
              fall *= by;
              l *= by;
              move = true;
              ref = m;
            }
          }
          // O in units of the new references (nothing is there before the first product)
          if (!(begin && h == 0) && __any_sync(0xffffffffu, move)) {
            // the product of the half before (the one before that is done: the step's scores came after it)
            TC_WAIT(sh.o_done[t][h ^ 1], ((it - 1) >> 1) & 1);
            tc::fence_after();
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
              uint32_t o[32];
              tc::tmem_ld32(o_at + 32 * c, o);
              wait_ld(o);
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * fall);
              tc::tmem_st32(o_at + 32 * c, o);
            }
          }
          const float base = ref == -INFINITY ? 0.f : ref;
#pragma unroll 1
          for (int q = 0; q < 2; ++q) {
            uint32_t v[32], pk[16];
            tc::tmem_ld32(s_at + 64 * h + 32 * q, v);
            wait_ld(v);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int g = 4 * h + 2 * q + e;
              const float f = fmaxf(st.ks[g] * qscale, kLeast), add = st.lr[g] - base;
              const float2 ff = make_float2(f, f), aa = make_float2(add, add);
              float2 sum = make_float2(0.f, 0.f);
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                float2 x2 = fma2(make_float2(__uint_as_float(v[16 * e + 2 * k]), __uint_as_float(v[16 * e + 2 * k + 1])), ff, aa);
                x2.x = fast_exp2(x2.x);
                x2.y = fast_exp2(x2.y);
                sum = add2(sum, x2);
                pk[8 * e + k] = pack_f16(x2.x, x2.y);
              }
              l = fmaf(sum.x + sum.y, st.rr[g], l);
            }
            tmem_st16(s_at + 64 * h + 16 * q, pk);  // (over scores that are in registers already)
          }
          tc::tmem_wait_st();
          tc::fence_before();
          tc::bar_arrive(&sh.p_full[t][h]);
        }
      }
      if (end) break;
      __syncwarp();
      if (lane == 0) tc::bar_arrive(&sh.step_free[n % kRing]);
      ++n;
    }

    // the row's result
    const bool done = x.ta == 0 && x.tb == x.tiles;
    const int slot = x.ta > 0 ? 0 : 1;
    const int tok = div_group(p, at);
    const int64_t to = (x.s.row0 + tok) * p.H + x.h * p.G + at - tok * p.G;
    const int64_t mypart = ((int64_t)blockIdx.x * 2 + slot) * kR + row;
    if (mine) {
      TC_WAIT(sh.o_done[t][1], ((it >> 1) - 1) & 1);
      tc::fence_after();
      float scale = l == 0.f ? 0.f : done ? rho / l : rho;
      float l2 = l == 0.f ? -INFINITY : ref + log2f(l), pre = 0.f;  // the prefix's weight
      uint16_t* out = p.out + to * D;
      float* part = p.part_o + mypart * D;
      const bool joins = P::mode == kTail && done && x.s.page0 > 0;  // (the same for all rows)
      const bool out16 = P::mode != kPrefix && done;                 // 16-bit results,
      const bool half_out = out16 && !joins;                         // and in shared memory too
      if constexpr (P::mode == kPrefix)
        if (done) part = p.pre_o + to * D;
      if constexpr (P::mode == kTail)
        if (joins && there) {
          float b;
          l2 = join_prefix(p, to, l2, pre, b);
          scale *= b;
        }
      // By way of the warp's own queries' place (they are done with), so that whole rows are
      // written at once: row r's 16-byte piece c lies where a query's would.
      constexpr int CH = D / 8, RPI = 32 / CH;  // pieces of a row there, rows of a write
      unsigned char* stage = q_smem + t * kK * D * 2;
      auto place = [&](int rr, int c) { return stage + (c >> 3) * 16384 + rr * 128 + (((c & 7) ^ (rr & 7)) << 4); };
      const int live = min(x.s.rows * p.G - (x.rt * kR + (row & ~31)), 32);  // rows of the warp
      const bool fits = !there || in_bounds(x.s.row0 + tok < p.total_rows && x.h * p.G + at - tok * p.G < p.H, p.c.status, kSiteAttendRow);
      const uint64_t mine_at = !fits ? 0 : out16 ? reinterpret_cast<uint64_t>(out) : reinterpret_cast<uint64_t>(part);
#pragma unroll 1
      for (int pass = 0; pass < (half_out ? 1 : 2); ++pass) {
        const int cols = half_out ? D : D / 2;
#pragma unroll 1
        for (int c = 0; c < cols; c += 16) {
          uint32_t o[16];
          tmem_ld16(o_at + pass * (D / 2) + c, o);
          float v[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = l == 0.f ? 0.f : __uint_as_float(o[k]) * scale;
          if (half_out) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
              *reinterpret_cast<uint4*>(place(r, c / 8 + k)) =
                  make_uint4(out_pair<BF16>(v[8 * k], v[8 * k + 1]), out_pair<BF16>(v[8 * k + 2], v[8 * k + 3]),
                             out_pair<BF16>(v[8 * k + 4], v[8 * k + 5]), out_pair<BF16>(v[8 * k + 6], v[8 * k + 7]));
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              *reinterpret_cast<float4*>(place(r, c / 4 + k)) = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
          }
        }
        __syncwarp();
        if constexpr (P::mode == kTail)
          if (joins) {  // four values of a row's tail, and of its prefix: eight rows' under way together
            constexpr int AHEAD = 8;
#pragma unroll 1
            for (int i0 = 0; i0 < 32 / RPI; i0 += AHEAD) {
              float4 y[AHEAD];
              int64_t first[AHEAD];
#pragma unroll
              for (int i = 0; i < AHEAD; ++i) {
                const int rr = (i0 + i) * RPI + lane / CH;
                const uint64_t to_at = __shfl_sync(0xffffffffu, mine_at, rr);
                const bool ok = rr < live && in_bounds(to_at != 0, p.c.status, kSiteAttendRow);
                first[i] = ok ? (int64_t)(to_at - reinterpret_cast<uint64_t>(p.out)) / 2 + pass * (D / 2) + lane % CH * 4 : -1;
                y[i] = ok ? __ldcg(reinterpret_cast<const float4*>(p.pre_o + first[i])) : make_float4(0.f, 0.f, 0.f, 0.f);
              }
#pragma unroll
              for (int i = 0; i < AHEAD; ++i) {
                const int rr = (i0 + i) * RPI + lane / CH;
                const float w = __shfl_sync(0xffffffffu, pre, rr);
                const float4 v = *reinterpret_cast<const float4*>(place((r & ~31) + rr, lane % CH));
                if (first[i] >= 0)
                  *reinterpret_cast<uint2*>(p.out + first[i]) =
                      make_uint2(out_pair<BF16>(fmaf(y[i].x, w, v.x), fmaf(y[i].y, w, v.y)),
                                 out_pair<BF16>(fmaf(y[i].z, w, v.z), fmaf(y[i].w, w, v.w)));
              }
            }
            __syncwarp();
            continue;
          }
#pragma unroll 4
        for (int i = 0; i < 32 / RPI; ++i) {
          const int rr = i * RPI + lane / CH, c = lane % CH;
          const uint64_t to_at = __shfl_sync(0xffffffffu, mine_at, rr);
          const uint4 v = *reinterpret_cast<const uint4*>(place((r & ~31) + rr, c));
          if (rr < live && in_bounds(to_at != 0, p.c.status, kSiteAttendRow)) reinterpret_cast<uint4*>(to_at)[pass * CH + c] = v;
        }
        __syncwarp();
      }
      if (there && fits && sh.any_nan[seg & 3]) {
#pragma unroll 1
        for (int d = 0; d < D; ++d)
          if (sh.nan_first[seg & 3][d] < limit) {
            if (out16)
              out[d] = BF16 ? 0x7fc0 : 0x7e00;
            else
              part[d] = __int_as_float(0x7fc00000);
          }
      }
      tc::fence_before();
      if (there && fits) {
        if (done) {
          if (P::mode == kPrefix)
            p.pre_l[to] = l2;
          else if (p.lse)
            p.lse[to] = l2 * 0.69314718056f;
        } else {
          p.part_ml[mypart] = make_float2(l == 0.f ? -INFINITY : ref, l);
        }
      }
    }
    if constexpr (P::mode == kPrefix) {
      // A prefix's parts are joined by a launch behind this one (join_kernel): an item may have a part in every
      // CTA, and one CTA alone would take longer over the sums than all of them over the products.
      if (threadIdx.x == 0 && x.ta == 0) {
        const int2 who = done ? make_int2(0, -1) : item_stretches<kOver>(sh.line, x);
        if (in_bounds(range_at(p, x) < p.range_tiles, p.c.status, kSiteAttendPart)) p.ranges[(int64_t)x.h * p.range_tiles + range_at(p, x)] = who;
      }
    } else if (!done) {
      TC_MEET();
      const int2 who = item_stretches<kOver>(sh.line, x);
      const int first = who.x, last = who.y;
      const bool fits = in_bounds(first >= 0 && first < last && last < sh.line.stretches && sh.line.stretches <= kAttendTcCtas &&
                                      (int)blockIdx.x >= first && (int)blockIdx.x <= last, p.c.status, kSiteAttendPart);
      if (threadIdx.x == 0) sh.last = fits && arrive_count(&p.counters[first]) == last - first;
      TC_MEET();
      if (sh.last) {
        if (mine) {
          // Lane l has row l's maximum, sum and weights; then the warp goes through its
          // rows, all lanes on one, the parts' loads in flight together. The weights are
          // in the place of the warp's own queries, 32 parts at a time.
          auto part = [&](int c, int rr) { return ((int64_t)c * 2 + (c == first ? 1 : 0)) * kR + t * 128 + (r & ~31) + rr; };
          float* wt = reinterpret_cast<float*>(q_smem + t * kK * D * 2 + (r & ~31) * 128);  // [32 parts][32 rows]
          const int rows = min(x.s.rows * p.G - (x.rt * kR + (row & ~31)), 32);
          float mx = -INFINITY, sum = 0.f;
          if (there) {
#pragma unroll 1
            for (int c = first; c <= last; ++c) mx = fmaxf(mx, __ldcg(&p.part_ml[part(c, lane)]).x);
          }
          const float base = mx == -INFINITY ? 0.f : mx;
          if (there) {
#pragma unroll 1
            for (int c = first; c <= last; ++c) {
              const float2 ml = __ldcg(&p.part_ml[part(c, lane)]);
              sum += ml.y * fast_exp2(ml.x - base);
            }
          }
          float inv = sum == 0.f ? 0.f : 1.f / sum, l2 = sum == 0.f ? -INFINITY : mx + log2f(sum), pre = 0.f;
          if (there && in_bounds(to < p.total_rows * p.H, p.c.status, kSiteAttendRow)) {
            if (P::mode == kTail && x.s.page0 > 0) {
              float b;
              l2 = join_prefix(p, to, l2, pre, b);
              inv *= b;
            }
            if (p.lse) p.lse[to] = l2 * 0.69314718056f;
          }
#pragma unroll 1
          for (int c0 = first; c0 <= last; c0 += 32) {
            const int n = min(last - c0 + 1, 32);
            __syncwarp();
#pragma unroll 1
            for (int k = 0; k < n; ++k)
              wt[k * 32 + lane] = there ? fast_exp2(__ldcg(&p.part_ml[part(c0 + k, lane)]).x - base) * inv : 0.f;
            __syncwarp();
            constexpr int V = D / 32, ROWS = 8;  // values a lane holds of a row, rows whose loads are in flight
#pragma unroll 1
            for (int r0 = 0; r0 < rows; r0 += ROWS) {
              float acc[ROWS][V];
#pragma unroll
              for (int i = 0; i < ROWS; ++i)
#pragma unroll
                for (int q = 0; q < V; ++q) acc[i][q] = 0.f;
#pragma unroll 1
              for (int k = c0 > first ? -1 : 0; k < n; ++k) {
                // (-1: the blocks before, kept in the first part's place)
                float v[ROWS][V];
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                  const float* from = p.part_o + part(k < 0 ? first : c0 + k, min(r0 + i, rows - 1)) * D + lane * V;
                  if constexpr (V == 4) {
                    const float4 y = __ldcg(reinterpret_cast<const float4*>(from));
                    v[i][0] = y.x, v[i][1] = y.y, v[i][2] = y.z, v[i][3] = y.w;
                  } else {
                    const float2 y = __ldcg(reinterpret_cast<const float2*>(from));
                    v[i][0] = y.x, v[i][1] = y.y;
                  }
                }
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                  const float w = k < 0 ? 1.f : wt[k * 32 + r0 + i];
#pragma unroll
                  for (int q = 0; q < V; ++q) acc[i][q] = fmaf(v[i][q], w, acc[i][q]);
                }
              }
#pragma unroll
              for (int i = 0; i < ROWS; ++i) {
                const float total = __shfl_sync(0xffffffffu, P::mode == kTail ? l2 : sum, (r0 + i) & 31);
                const uint64_t row_to = __shfl_sync(0xffffffffu, (uint64_t)to, (r0 + i) & 31);
                const float row_pre = P::mode == kTail ? __shfl_sync(0xffffffffu, pre, (r0 + i) & 31) : 0.f;
                if (r0 + i < rows && in_bounds((int64_t)row_to < p.total_rows * p.H, p.c.status, kSiteAttendRow)) {
                  if (c0 + n <= last) {
                    float* keep = p.part_o + part(first, r0 + i) * D + lane * V;
#pragma unroll
                    for (int q = 0; q < V; ++q) keep[q] = acc[i][q];
                  } else {
                    const bool none = P::mode == kTail ? total == -INFINITY : total == 0.f;
                    if (P::mode == kTail && row_pre != 0.f) {
                      const float* pre_o = p.pre_o + row_to * D + lane * V;
#pragma unroll
                      for (int q = 0; q < V; ++q) acc[i][q] = fmaf(__ldcg(pre_o + q), row_pre, acc[i][q]);
                    }
                    uint32_t* out = reinterpret_cast<uint32_t*>(p.out + row_to * D + lane * V);
#pragma unroll
                    for (int q = 0; q < V; q += 2) out[q / 2] = none ? 0u : out_pair<BF16>(acc[i][q], acc[i][q + 1]);
                  }
                }
              }
            }
          }
        }
      }
    }
    // (the segment's last record is given back once its notes have been read)
    __syncwarp();
    if (lane == 0) tc::bar_arrive(&sh.step_free[n % kRing]);
    ++n;
    ++seg;
  } while (walk_next<kR, kK, kOver>(p, sh, x));
}

// A wait that ran out leaves items without their last arrival, so the last CTA to leave clears
// the counters whatever they are: the next call on the workspace has to find zeros.
// count_out: by the thread that makes the CTA's arrivals, after the last of them; true for the last CTA.
// (Relaxed: the arrivals have returned their counts by then. And not at the very end, where its way
// through the busy memory system is waited for: 4 us of a prefix of 8,257 tokens.)
__device__ __forceinline__ int count_out(const AttendParams& p, int stretches) {
  return atomicAdd(&p.counters[kAttendCtas], 1) == stretches - 1;
}
__device__ __forceinline__ void clear_counters(const AttendParams& p) {
  static_assert(kAttendCtas <= kThreads, "a counter a thread");
  if (threadIdx.x < kAttendCtas) p.counters[threadIdx.x] = 0;
  if (threadIdx.x == 0) p.counters[kAttendCtas] = 0;
}

template <int D, bool BF16, int MODE>
__global__ void __launch_bounds__(kThreads, 1)
    attend_tc_kernel(AttendCall<MODE> p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  constexpr int kBytes = kK * D * 2;
  // queries 2 tiles, keys and values 2 stages each, codes as they come: 7 x 32 KB (D = 128)
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* q_smem = smem;
  unsigned char* k_smem = smem + 2 * kBytes;
  unsigned char* v_smem = smem + 4 * kBytes;
  unsigned char* raw = smem + 6 * kBytes;
  Shared& sh = *reinterpret_cast<Shared*>(smem + 7 * kBytes);
  int64_t* scan = reinterpret_cast<int64_t*>(&sh.nan_first[0][0]);
  const int warp = threadIdx.x >> 5;
  pdl_wait();
  Line line;
  const LinePart part = attend_line<kR, kK, kOver, kThreads>(p, kOver + 1, scan, line);
  if (line.units == 0 || (int)blockIdx.x >= line.stretches) return;
  Stretch w;
  attend_find<kR, kK, kOver, kThreads>(p, line, part, blockIdx.x, scan, w);
  {
    Walk x;
    if (!walk_begin<kR, kK, kOver>(p, w, x)) {  // no tile in the stretch: every role has at least one from here on
      if (threadIdx.x == 0) sh.left = count_out(p, line.stretches);
      __syncthreads();
      if (sh.left) clear_counters(p);
      return;
    }
  }
  if (threadIdx.x == 0) {
    sh.u0 = w.u0;
    sh.u1 = w.u1;
    sh.line = line;
    sh.seq = w.seq;
    sh.head = w.head;
    sh.row_tile = w.row_tile;
    sh.in_item = w.in_item;
    sh.stop = 0;
    tc::bar_init(&sh.meet, 256);
    tc::bar_init(&sh.drain, 2);
    for (int k = 0; k < 2; ++k) {
      tc::bar_init(&sh.q_full[k], 128);
      tc::bar_init(&sh.k_full[k], 128);
      tc::bar_init(&sh.v_full[k], 128);
      tc::bar_init(&sh.k_free[k], 2);
      tc::bar_init(&sh.v_free[k], 2);
      for (int h = 0; h < 2; ++h) {
        tc::bar_init(&sh.s_full[k][h], 1);
        tc::bar_init(&sh.p_full[k][h], 128);
        tc::bar_init(&sh.o_done[k][h], 1);
      }
      tc::bar_init(&sh.raw_full[k], 1);
      tc::bar_init(&sh.raw_free[k], 4);
    }
    for (int k = 0; k < kRing; ++k) {
      tc::bar_init(&sh.step_full[k], 1);
      tc::bar_init(&sh.step_free[k], 14);  // every warp that reads it
    }
    tc::bar_fence_init();
  }
  __syncthreads();
  if (threadIdx.x < 4) sh.any_nan[threadIdx.x] = 0;
  for (int d = threadIdx.x; d < 4 * 128; d += kThreads) (&sh.nan_first[0][0])[d] = 0x7fffffff;
  if (warp == 12) tc::tmem_alloc(&sh.tmem, 512);
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  const uint32_t tmem = sh.tmem;
  // registers: 512 threads start with 128 each, four warpgroups split them
  if (warp < 8) {
    tc::setmaxnreg_inc<kRegSoftmax>();
    softmax_role<D, BF16>(p, sh, q_smem, tmem, warp >> 2);
    if (threadIdx.x == 0) sh.left = count_out(p, sh.line.stretches);
  } else if (warp < 12) {
    tc::setmaxnreg_dec<kRegConvert>();
    convert_role<D>(p, sh, k_smem, v_smem, raw);
  } else {
    tc::setmaxnreg_dec<kRegIssue>();
    if (warp == 12 || warp == 14)
      mma_role<D>(p, sh, tc::su32(q_smem), tc::su32(k_smem), tc::su32(v_smem), tmem, warp == 14);
    else if (warp == 13)
      plan_role<D>(p, sh, map_k, map_v, raw);
  }
  __syncthreads();
  // after a wait that ran out, products and copies may still be in flight (the lane that issued the
  // products is the one whose commit covers them)
  if (sh.stop && (warp == 12 || warp == 14) && elect_one()) {
    tc::mma_commit(&sh.drain);
    tc::bar_wait(&sh.drain, 0, nullptr, kWaitNs);
    for (int k = 0; k < 2; ++k) {
      tc::bar_wait(&sh.raw_full[k], 0, nullptr, kWaitNs / 8);
      tc::bar_wait(&sh.raw_full[k], 1, nullptr, kWaitNs / 8);
    }
  }
  __syncthreads();
  if (sh.left) clear_counters(p);
  if (warp == 12) tc::tmem_dealloc(tmem, 512);
}

// The parts that a prefix's items left, a warp a row: its maximum, weights and sums. A CTA takes kJoinRows rows of an
// item; grid: y over key heads, z over groups.
constexpr int kJoinRows = 8;
template <int D>
__global__ void __launch_bounds__(256) join_kernel(AttendCall<kPrefix> p) {
  pdl_wait();
  const SeqInfo s = attend_seq(p, blockIdx.z);
  const int lane = threadIdx.x & 31, h = blockIdx.y, rows = s.rows * p.G;
  constexpr int V = D / 32;
  for (int r0 = blockIdx.x * kJoinRows; r0 < rows; r0 += gridDim.x * kJoinRows) {
    const int tile = range_at(p, s.row0, blockIdx.z, r0 / kR);
    if (!in_bounds(tile < p.range_tiles, p.c.status, kSiteAttendPart)) continue;
    const int2 who = p.ranges[(int64_t)h * p.range_tiles + tile];
    // one part: it is the result. (Whatever is there where the items were given up, which is recorded: no part to join.)
    if (who.y <= who.x || who.x < 0 || who.y >= kAttendTcCtas) continue;
    const int n = who.y - who.x + 1;
    for (int at = r0 + (threadIdx.x >> 5); at < min(r0 + kJoinRows, rows); at += 8) {
      auto part = [&](int c) { return ((int64_t)(who.x + c) * 2 + (c == 0 ? 1 : 0)) * kR + at % kR; };
      float2 ml[kAttendTcCtas / 32];
      float mx = -INFINITY, sum = 0.f;
#pragma unroll
      for (int k = 0; k < kAttendTcCtas / 32; ++k) {
        ml[k] = k * 32 + lane < n ? p.part_ml[part(k * 32 + lane)] : make_float2(-INFINITY, 0.f);
        mx = fmaxf(mx, ml[k].x);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float base = mx == -INFINITY ? 0.f : mx;
#pragma unroll
      for (int k = 0; k < kAttendTcCtas / 32; ++k) {
        ml[k].x = fast_exp2(ml[k].x - base);
        sum = fmaf(ml[k].y, ml[k].x, sum);
      }
      sum = warp_sum(sum);
      float acc[V];
#pragma unroll
      for (int q = 0; q < V; ++q) acc[q] = 0.f;
#pragma unroll
      for (int k = 0; k < kAttendTcCtas / 32; ++k) {
#pragma unroll 1
        for (int c0 = 0; c0 < min(n - k * 32, 32); c0 += 16) {
          alignas(16) float y[16][V];  // (all of them under way together)
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const float* from = p.part_o + part(min(k * 32 + c0 + c, n - 1)) * D + lane * V;
            if constexpr (V == 4)
              *reinterpret_cast<float4*>(y[c]) = *reinterpret_cast<const float4*>(from);
            else
              *reinterpret_cast<float2*>(y[c]) = *reinterpret_cast<const float2*>(from);
          }
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const float w = __shfl_sync(0xffffffffu, ml[k].x, c0 + c);  // (0 past the last part)
#pragma unroll
            for (int q = 0; q < V; ++q) acc[q] = fmaf(y[c][q], k * 32 + c0 + c < n ? w : 0.f, acc[q]);
          }
        }
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const int j = div_group(p, at);
      const int64_t to = (s.row0 + j) * p.H + h * p.G + at - j * p.G;
      if (!in_bounds(to < p.total_rows * p.H, p.c.status, kSiteAttendRow)) continue;
#pragma unroll
      for (int q = 0; q < V; ++q) p.pre_o[to * D + lane * V + q] = sum == 0.f ? 0.f : acc[q] * inv;
      if (lane == 0) p.pre_l[to] = sum == 0.f ? -INFINITY : mx + log2f(sum);
    }
  }
}

// Once per device: the shared memory, and that the register split adds up --
// setmaxnreg.inc waits for registers that only the launch's own can give.
template <int D, bool BF16, int MODE>
int prepare(int smem) {
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return OCCAM_ERR_CUDA;
  if ((ready.load(std::memory_order_acquire) >> dev) & 1) return OCCAM_OK;
  cudaFuncAttributes at;
  if (cudaFuncGetAttributes(&at, attend_tc_kernel<D, BF16, MODE>) != cudaSuccess) return OCCAM_ERR_CUDA;
  if (at.numRegs * kThreads < 256 * kRegSoftmax + 128 * (kRegConvert + kRegIssue)) return OCCAM_ERR_UNSUPPORTED;
  if (cudaFuncSetAttribute(attend_tc_kernel<D, BF16, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
    return OCCAM_ERR_CUDA;
  ready.fetch_or(uint64_t(1) << dev, std::memory_order_release);
  return OCCAM_OK;
}

template <int D, bool BF16, int MODE>
int launch(const AttendCall<MODE>& p, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t st) {
  const int smem = 7 * kK * D * 2 + kSharedBytes;
  const int rc = prepare<D, BF16, MODE>(smem);
  if (rc != OCCAM_OK) return rc;
  const dim3 grid((unsigned)std::min(cache_sms(), kAttendTcCtas));
  return launch_after(attend_tc_kernel<D, BF16, MODE>, grid, kThreads, smem, st, p, mk, mv) && cudaGetLastError() == cudaSuccess
             ? OCCAM_OK
             : OCCAM_ERR_CUDA;
}

}  // namespace

template <int MODE>
int occam::launch_attend_tc(const AttendCall<MODE>& p, int dim, cudaStream_t st) {
  CUtensorMap mk, mv;
  if (!encode_blocks(&mk, p.c, p.c.k, dim, p.c.T, false) || !encode_blocks(&mv, p.c, p.c.v, dim, p.c.T, false))
    return OCCAM_ERR_CUDA;
  const int rc = dim == 128 ? (p.bf16 ? launch<128, true>(p, mk, mv, st) : launch<128, false>(p, mk, mv, st))
                            : (p.bf16 ? launch<64, true>(p, mk, mv, st) : launch<64, false>(p, mk, mv, st));
  if constexpr (MODE == kPrefix) {
    if (rc != OCCAM_OK) return rc;
    static_assert(kAttendTcCtas % 32 == 0, "parts a lane");
    // (eight CTAs an SM; more of them, most with nothing to join, took 17 us)
    const int64_t want = p.total_rows * p.G / p.n / kJoinRows + 1, most = cache_sms() * 8 / ((int64_t)p.c.heads * p.n);
    const dim3 grid((unsigned)std::max<int64_t>(std::min(want, most), 1), (unsigned)p.c.heads, (unsigned)p.n);
    const bool ok = dim == 128 ? launch_after(join_kernel<128>, grid, 256, 0, st, p) : launch_after(join_kernel<64>, grid, 256, 0, st, p);
    return ok && cudaGetLastError() == cudaSuccess ? OCCAM_OK : OCCAM_ERR_CUDA;
  }
  return rc;
}
template int occam::launch_attend_tc<kWhole>(const AttendCall<kWhole>&, int, cudaStream_t);
template int occam::launch_attend_tc<kPrefix>(const AttendCall<kPrefix>&, int, cudaStream_t);
template int occam::launch_attend_tc<kTail>(const AttendCall<kTail>&, int, cudaStream_t);
