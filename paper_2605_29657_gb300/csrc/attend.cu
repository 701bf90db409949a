// attend.cu -- attention over the paged 8-bit cache for few query rows per key
// head (single tokens, a few speculative ones), and the C-ABI entry.
//
// With m the running maximum of s_k = scale * s(q) * ks(k) * (q . codes_k),
// in log2 units, one pass keeps l = sum 2^(s_k - m) and O = sum 2^(s_k - m) v_k
// and rescales both when m grows. Bound by HBM: the codes are read once, 1
// byte a value (64 tokens over ragged caches, 301 MB: 65 us, 4.9 TB/s; 4 tokens over
// 16 k tokens of 32 heads, 544 MB: 102 us, 5.3 TB/s), and for small caches by the chain
// from lengths over tables and codes to the join (612 tokens: 9 us). Each
// warp runs its own key tiles of 32 keys with no barrier between them; two tiles'
// copies to shared memory are always under way.
//  - S^T = K Q^T and O^T = V^T P^T (m16n8k16, f16 operands, fp32 sums): keys and
//    dims fill the 16 rows, up to 8 query rows the 8 columns, so one token of a
//    group of 8 heads wastes nothing. The order of the summed index is free, so
//    each lane's 16 bytes of a key row are the operands of four steps as
//    they come; v's codes of two keys are interleaved by byte permutes; P is
//    transposed by movmatrix.
//  - e4m3 codes convert to f16 exactly. Query rows are brought to f16 by a power of two of
//    their own (bf16's 8 bits fit; what falls below 2^-38 of a row's largest
//    value is lost), undone in fp32.
//  - a NaN value counts for the rows that see its token only: in tiles that
//    some row does not see whole, NaN codes are left out of the product and the
//    first such token of each dim is noted for the rows past it.
//  - the scales of v enter P relative to a running reference, so that P stays
//    in f16's range whatever the scales are. P's rounding to f16 (11 bits) is of the size of
//    an f16 result's own: against 64 bits 2.5e-4 where fp32 throughout gives 2.1e-4 (4 videos,
//    f16 results), with bf16 results 1.6e-3 either way. l is the sum of the unrounded P.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "attend.cuh"
#include "attend_tc.cuh"
#include "nvtx.cuh"

using namespace occam;

namespace {

constexpr int kTile = 32;   // keys of a unit
// What beginning and ending an item costs, in units (64 single tokens, 37 k units:
// 3: 80 us, 8: 69, 16: 65, 32: 67, 48: 74; the first copies' way through
// the busy memory system is most of it).
constexpr int kOver = 16;
constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
// Query rows of a key head this file's kernel is used for. Caches of 2,300 tokens, 8
// key heads; here / on tcgen05 (whose tile has 256 rows whatever is in them):
// 64 sequences 8 rows 69 / 176 us, 16: 98 / 179, 32: 171 / 180, 48: 237 / 181;
// 8 sequences 16 rows 27 / 42 us, 32: 37 / 42, 48: 46 / 42.
constexpr int kFewRows = 32;
constexpr float kRhoKeep = 1.f / 64.f;           // P is scaled down by v's scales at most this far
constexpr float kRhoSpan = 8.6736174e-19f;       // 2^-60
// P (at most 1) goes to f16 2^15 times as large: what is 2^-29 of a row's running maximum still has
// f16's 11 bits, below 2^-40 it is lost. (As it is, 2^-14 and 2^-25: a long cache's many small
// probabilities were missing from O, while l, summed in fp32, had them.)
constexpr float kLift = 32768.f, kUnlift = 1.f / 32768.f;

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float q_value(uint16_t x, int bf16) {
  return bf16 ? __uint_as_float((uint32_t)x << 16) : __half2float(__ushort_as_half(x));
}
__device__ __forceinline__ uint16_t out_bits(float x, int bf16) {
  return bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(x)) : __half_as_ushort(__float2half_rn(x));
}

// Rows of 128 (64) bytes lie in shared memory with the 128-byte (64-byte) swizzle.
// piece: where a row's 16-byte piece c is. order: the rows and pieces that
// neighbouring lanes take, so that eight lanes always meet eight different banks' groups.
template <int D>
__device__ __forceinline__ int piece(int row, int c) { return D == 128 ? c ^ (row & 7) : c ^ ((row >> 1) & 3); }
template <int D>
__device__ __forceinline__ int order(int g) { return D == 128 ? (g >> 1) | ((g & 1) << 2) : g; }
template <int D>
__device__ __forceinline__ int value_place(int row, int g) {
  return D == 128 ? piece<D>(row, order<D>(g)) * 16 : piece<D>(row, g >> 1) * 16 + (g & 1) * 8;
}
// 16 bytes from global to shared memory, zeros if !there
__device__ __forceinline__ void copy_async16(uint32_t dst, const uint8_t* src, uint32_t there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
// a box of rows of page `page` (of all layers) from row `row` (of all heads) on
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, int row, int page, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(0), "r"(row), "r"(page), "r"(smem_u32(bar))
      : "memory");
}
template <int WORDS>
__device__ __forceinline__ void read_codes(uint32_t (&r)[WORDS], uint32_t src) {
  if constexpr (WORDS == 4)
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(src) : "memory");
  else
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(src) : "memory");
}

// A key tile's place: known one tile before its copies are issued
struct TileMeta {
  int page[2];    // of each 16 keys
  uint32_t seen;  // bit k: key k of the tile may be seen (before settle(): this lane's flag)
};
// What the products need of a tile whose copies are under way
struct TileScales {
  uint32_t seen;
  float ks[2], vs[2];
};

// Takes NaN codes (of either sign) out of a word of values of one key, dims d .. d+3, and
// notes the key as the first of those dims.
__device__ __forceinline__ void note_nans(uint32_t& w, int key, int d, int* first) {
  const uint32_t hit = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  if (hit) {
#pragma unroll
    for (int b = 0; b < 4; ++b)
      if ((hit >> (8 * b + 7)) & 1) {
        atomicMin(&first[d + b], key);
        w &= ~(0xffu << (8 * b));
      }
  }
}

// NQ: tiles of 8 query rows. TMA: whole tiles come by tensor copies; else row by
// row, leaving out hidden rows.
template <int D, int NQ, bool TMA>
__global__ void __launch_bounds__(kThreads, NQ == 1 ? 3 : 2)
    attend_rows_kernel(AttendParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  constexpr int R = 8 * NQ;
  constexpr int KC = D / 64;      // 16-byte pieces of a key row a lane holds
  constexpr int VW = D / 32;      // 4-byte words of a value row a lane holds
  constexpr int MT = D / 16;      // tiles of 16 dims
  __shared__ int64_t sh[kWarps + 4];
  __shared__ float sh_m[kWarps][R], sh_l[kWarps][R];
  __shared__ int sh_last;
  __shared__ int sh_nan[2][D];  // first token with a NaN in that dim, of those taken out; by turns of segments
  // Each warp's copies: two slots of keys and two of values, 32 rows each. At the end
  // of a segment the warp's sums take their place.
  constexpr int kSlot = kTile * D, kWarpBytes = 4 * kSlot;
  static_assert(kWarpBytes >= R * D * 4, "a warp's sums fit its copies' place");
  __shared__ uint64_t sh_bar[kWarps][4];
  extern __shared__ __align__(1024) unsigned char sh_dyn[];
  unsigned char* sh_slots = sh_dyn + ((1024 - (smem_u32(sh_dyn) & 1023)) & 1023);
  float* sh_o = reinterpret_cast<float*>(sh_slots);       // row r of warp w: (w kWarpBytes / 4) + r D
  constexpr int kWarpFloats = kWarpBytes / 4;

  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  const uint32_t k_at = smem_u32(sh_slots) + warp * kWarpBytes, v_at = k_at + 2 * kSlot;
  uint64_t* bars = sh_bar[warp];  // keys of slot 0, 1, values of slot 0, 1
  uint32_t turn = 0;              // tiles this warp has taken
  if (TMA && threadIdx.x < kWarps * 4) mbar_init(&sh_bar[0][0] + threadIdx.x, 1);
  if (TMA) fence_mbar_init();
  for (int d = threadIdx.x; d < 2 * D; d += kThreads) sh_nan[0][d] = 0x7fffffff;
  pdl_wait();
  Line line;
  // (a stretch has a tile a warp at least: one sequence of 2,300 tokens takes 12.5 us, with two
  // tiles a warp 13.6, with five 17.8)
  const LinePart mine = attend_line<R, kTile, kOver, kThreads>(p, kWarps, sh, line);
  if (line.units == 0 || (int)blockIdx.x >= line.stretches) return;
  Stretch w;
  attend_find<R, kTile, kOver, kThreads>(p, line, mine, blockIdx.x, sh, w);
  Walk x0;
  if (!walk_begin<R, kTile, kOver>(p, w, x0)) return;
  int* nan_first = sh_nan[0];
  do {
    const SeqInfo s = x0.s;
    const int i = x0.i, h = x0.h, rt = x0.rt, tiles = x0.tiles, ta = x0.ta, tb = x0.tb;
    const int rows = s.rows * p.G - rt * R;  // rows of this tile that exist, from 0
    const int32_t* table = p.c.table + (int64_t)s.seq * p.c.max_pages;
    const uint8_t* flags = nullptr;
    int n_flags = 0;
    if (p.keep) {
      const int64_t k0 = p.keep_off[i], k1 = p.keep_off[i + 1];
      if (k0 >= 0 && k1 >= k0 && k1 <= p.total_keep) {
        flags = p.keep + k0;
        n_flags = (int)min(k1 - k0, (int64_t)s.len);
      } else {
        set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
      }
    }

    const int64_t layer_page = (int64_t)p.layer * p.c.pages;
    const int tmask = p.c.T - 1;
    auto meta_of = [&](int tile) {
      TileMeta x;
      const int key = tile * kTile;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int first = key + 16 * k;
        const bool there = first < s.len && in_bounds((first >> p.c.log2T) < p.c.max_pages, p.c.status, kSiteAttendKey);
        x.page[k] = there ? table[first >> p.c.log2T] : 0;
      }
      bool see = key + lane < s.len;
      if (key + lane < n_flags && in_bounds(flags + key + lane < p.keep + p.total_keep, p.c.status, kSiteAttendKey))
        see = flags[key + lane] != 0;
      x.seen = see;
      return x;
    };
    // the ballot is taken one tile later, when the flag has arrived
    auto settle = [&](TileMeta& x) {
      x.seen = __ballot_sync(0xffffffffu, x.seen != 0);
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if ((unsigned)x.page[k] >= (unsigned)p.c.pages) {
          set_status(p.c.status, OCCAM_ERR_INVALID_ARG);
          x.page[k] = 0;
          x.seen &= k ? 0x0000ffffu : 0xffff0000u;
        }
    };
    auto scales = [&](const TileMeta& x) {
      TileScales r;
      r.seen = x.seen;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int64_t b = (layer_page + x.page[k]) * p.c.heads + h;
        r.ks[k] = p.c.k_scale[b];
        r.vs[k] = p.c.v_scale[b];
      }
      return r;
    };
    // 32 rows of codes (keys or values) of a tile to the slot at `dst`
    auto copy = [&](const CUtensorMap& map, const uint8_t* codes, const TileMeta& x, int tile, uint32_t dst, uint64_t* bar) {
      if constexpr (TMA) {
        if (lane == 0) {
          if (p.c.T >= kTile) {
            mbar_arrive_expect_tx(bar, kTile * D);
            tma_rows(dst, &map, h * p.c.T + ((tile * kTile) & tmask), (int)layer_page + x.page[0], bar);
          } else {
            const bool both = (x.seen >> 16) != 0;  // else the second page may not be there
            mbar_arrive_expect_tx(bar, both ? kTile * D : 16 * D);
#pragma unroll
            for (int k = 0; k < 2; ++k)
              if (k == 0 || both)
                tma_rows(dst + k * 16 * D, &map, h * p.c.T, (int)layer_page + x.page[k], bar);
          }
        }
      } else {
        // a lane takes a 16-byte piece of every RPC-th row; hidden rows are not read, but become zeros
        constexpr int LPR = D / 16, RPC = 32 / LPR;
        const int r0 = lane / LPR, c = lane % LPR;
#pragma unroll
        for (int i = 0; i < LPR; ++i) {
          const int row = i * RPC + r0;
          const int64_t b = (layer_page + (row < 16 ? x.page[0] : x.page[1])) * p.c.heads + h;
          copy_async16(dst + row * D + piece<D>(row, c) * 16, codes + ((b << p.c.log2T) + ((tile * kTile + row) & tmask)) * D + c * 16,
                       (x.seen >> row) & 1);
        }
        cp_async_commit();
      }
    };
    auto arrived = [&](uint64_t* bar) {
      if constexpr (TMA) {
        if (!mbar_wait(bar, (turn >> 1) & 1, kSpinLimit)) set_status(p.c.status, OCCAM_ERR_TIMEOUT);
      } else {
        cp_async_wait<3>();
      }
      __syncwarp();
    };

    // Two tiles' copies are under way ahead of the one in hand, keys and values
    // each by themselves.
    int tile = ta + warp;
    TileScales cur, nxt, far;
    TileMeta ahead;
    const int end = tb - 1;
    auto fetch = [&](int to) {
      TileMeta x = ahead;
      settle(x);
      ahead = meta_of(min(to + kWarps, end));
      return x;
    };
    if (tile < tb) {
      ahead = meta_of(tile);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int to = tile + i * kWarps;
        const TileMeta x = fetch(min(to, end));
        if (i == 0) cur = scales(x); else nxt = scales(x);
        const int slot = (turn + i) & 1;
        if (to < tb || !TMA) {
          TileMeta y = x;
          if (to >= tb) y.seen = 0;
          copy(map_k, p.c.k, y, min(to, end), k_at + slot * kSlot, bars + slot);
          copy(map_v, p.c.v, y, min(to, end), v_at + slot * kSlot, bars + 2 + slot);
        }
      }
    }
    // (while the first copies are under way) the query rows as f16, scaled by a power of two each
    uint32_t qf[NQ][4 * KC][2];
    float qscale[NQ][2];  // of rows 2t and 2t + 1
    int limit[NQ][2];     // keys those rows see
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int r = nq * 8 + g;
      float x[KC][16];
      float amax = 0.f;
      const int row = rt * R + r, j = div_group(p, row);
      const uint16_t* q = p.q + (s.row0 + j) * p.q_row + (int64_t)(h * p.G + row - j * p.G) * D;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        uint4 v[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        if (r < rows && in_bounds(s.row0 + j < p.total_rows && h * p.G + row - j * p.G < p.H, p.c.status, kSiteAttendRow)) {
          v[0] = *reinterpret_cast<const uint4*>(q + (t + 4 * c) * 16);
          v[1] = *reinterpret_cast<const uint4*>(q + (t + 4 * c) * 16 + 8);
        }
        const uint16_t* b = reinterpret_cast<const uint16_t*>(v);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          x[c][k] = q_value(b[k], p.bf16);
          amax = fmaxf(amax, finite_abs(x[c][k]));
        }
      }
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      // largest value in [2^14, 2^15): far from f16's end, small values far from its lower end
      int e = (__float_as_int(amax) >> 23) - 127 - 14;
      e = amax == 0.f ? 0 : max(e, -112);
      const float up = __int_as_float((127 - e) << 23);
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          qf[nq][c * 4 + k][0] = pack_f16(x[c][4 * k] * up, x[c][4 * k + 1] * up);
          qf[nq][c * 4 + k][1] = pack_f16(x[c][4 * k + 2] * up, x[c][4 * k + 3] * up);
        }
      const float down = __int_as_float((127 + e) << 23) * p.scale_log2;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        qscale[nq][k] = __shfl_sync(0xffffffffu, down, (2 * t + k) * 4);
        const int rr = nq * 8 + 2 * t + k;
        limit[nq][k] = rr >= rows ? 0 : p.causal ? s.len - s.rows + div_group(p, rt * R + rr) + 1 : s.len;
      }
    }
    // keys that every row of the tile sees
    const int common = p.causal ? s.len - s.rows + div_group(p, rt * R) + 1 : s.len;

    float o[NQ][MT][4], m[NQ][2], l[NQ][2];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
#pragma unroll
      for (int k = 0; k < MT; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nq][k][e] = 0.f;
      m[nq][0] = m[nq][1] = -INFINITY;
      l[nq][0] = l[nq][1] = 0.f;
    }
    float rho = 0.f, rho_max = 0.f;  // O is held in units of rho / kLift

    for (; tile < tb; tile += kWarps) {
      const int later = tile + 2 * kWarps;
      const int slot = turn & 1;
      TileMeta x2 = fetch(min(later, end));
      if (later >= tb) x2.seen = 0;
      // scores
      arrived(bars + slot);
      float sc[NQ][2][4];
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[nq][k][e] = 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          uint32_t kr[2][4];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int row = 16 * k + 8 * r + order<D>(g);
            read_codes<4>(kr[r], k_at + slot * kSlot + row * D + piece<D>(row, t + 4 * c) * 16);
          }
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint32_t lo = kr[0][x], hi = kr[1][x];
            const uint32_t a0 = e4m3x2_f16x2(lo), a2 = e4m3x2_f16x2_hi(lo);
            const uint32_t a1 = e4m3x2_f16x2(hi), a3 = e4m3x2_f16x2_hi(hi);
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) mma_f16(sc[nq][k], a0, a1, a2, a3, qf[nq][c * 4 + x][0], qf[nq][c * 4 + x][1]);
          }
        }
      const uint32_t seen = cur.seen;
      far = scales(x2);
      __syncwarp();
      if (later < tb || !TMA) copy(map_k, p.c.k, x2, min(later, end), k_at + slot * kSlot, bars + slot);
      // softmax: lane holds rows 2t, 2t + 1 of keys g, g + 8 of each 16
      const bool open = seen == 0xffffffffu && (tile + 1) * kTile <= common;
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[nq][k][e] *= cur.ks[k] * qscale[nq][e & 1];
        if (!open) {
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int key = 16 * k + 8 * (e >> 1) + order<D>(g);
              const bool see = ((seen >> key) & 1) && tile * kTile + key < limit[nq][e & 1];
              sc[nq][k][e] = see ? sc[nq][k][e] : -INFINITY;
            }
        }
        float grow[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = fmaxf(fmaxf(sc[nq][0][e], sc[nq][0][e + 2]), fmaxf(sc[nq][1][e], sc[nq][1][e + 2]));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
          const float mn = fmaxf(m[nq][e], x);
          const float ref = mn == -INFINITY ? 0.f : mn;  // nothing seen yet: every p is 0
          grow[e] = fast_exp2(m[nq][e] - ref);
          m[nq][e] = mn;
          l[nq][e] *= grow[e];
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              const float pr = fast_exp2(sc[nq][k][e + 2 * b] - ref);
              sc[nq][k][e + 2 * b] = pr;
              l[nq][e] += pr;
            }
        }
        if (__any_sync(0xffffffffu, grow[0] != 1.f || grow[1] != 1.f)) {
#pragma unroll
          for (int k = 0; k < MT; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nq][k][e] *= grow[e & 1];
        }
      }
      arrived(bars + 2 + slot);
      // O^T += V^T P^T, 16 keys at a time
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if ((seen >> (16 * k)) & 0xffff) {
          const float v = cur.vs[k];
          uint32_t vr[4][VW];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int row = 16 * k + 8 * (r >> 1) + order<D>(2 * t + (r & 1));
            read_codes<VW>(vr[r], v_at + slot * kSlot + row * D + value_place<D>(row, g));
            if (!open) {
              // hidden rows may be anything
#pragma unroll
              for (int x = 0; x < VW; ++x) {
                if (!((seen >> row) & 1)) vr[r][x] = 0;
                note_nans(vr[r][x], tile * kTile + row, order<D>(g) * (4 * VW) + 4 * x, nan_first);
              }
            }
          }
          if (v > rho || v < rho * kRhoKeep) {  // the same in every lane
            float to = v > rho ? v : fmaxf(v, rho_max * kRhoSpan);
            if (to != rho && to > 0.f) {
              const float f = rho / to;
#pragma unroll
              for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                for (int x = 0; x < MT; ++x)
#pragma unroll
                  for (int e = 0; e < 4; ++e) o[nq][x][e] *= f;
              rho = to;
              rho_max = fmaxf(rho_max, to);
            }
          }
          const float ratio = rho > 0.f ? v / rho * kLift : 0.f;
          uint32_t b0[NQ], b1[NQ];
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq) {
            b0[nq] = transpose8x8(pack_f16(sc[nq][k][0] * ratio, sc[nq][k][1] * ratio));
            b1[nq] = transpose8x8(pack_f16(sc[nq][k][2] * ratio, sc[nq][k][3] * ratio));
          }
#pragma unroll
          for (int x = 0; x < VW; ++x) {
            const uint32_t w0 = vr[0][x], w1 = vr[1][x], w2 = vr[2][x], w3 = vr[3][x];
            // two keys' bytes 0, 1 and 2, 3 side by side
            const uint32_t p0 = __byte_perm(w0, w1, 0x5140), p1 = __byte_perm(w0, w1, 0x7362);
            const uint32_t p2 = __byte_perm(w2, w3, 0x5140), p3 = __byte_perm(w2, w3, 0x7362);
            const uint32_t a0 = e4m3x2_f16x2(p0), a1 = e4m3x2_f16x2_hi(p0), a2 = e4m3x2_f16x2(p2), a3 = e4m3x2_f16x2_hi(p2);
            const uint32_t c0 = e4m3x2_f16x2(p1), c1 = e4m3x2_f16x2_hi(p1), c2 = e4m3x2_f16x2(p3), c3 = e4m3x2_f16x2_hi(p3);
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) {
              mma_f16(o[nq][2 * x], a0, a1, a2, a3, b0[nq], b1[nq]);
              mma_f16(o[nq][2 * x + 1], c0, c1, c2, c3, b0[nq], b1[nq]);
            }
          }
        }
      }
      __syncwarp();
      if (later < tb || !TMA) copy(map_v, p.c.v, x2, min(later, end), v_at + slot * kSlot, bars + 2 + slot);
      cur = nxt;
      nxt = far;
      ++turn;
    }
    if (!TMA) cp_async_wait<0>();

    // the warps' results meet in shared memory (every lane's copies have been read)
    __syncwarp();
    auto value = [&](float x) { return x * kUnlift * rho; };
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = l[nq][e];
        x += __shfl_xor_sync(0xffffffffu, x, 4);
        x += __shfl_xor_sync(0xffffffffu, x, 8);
        x += __shfl_xor_sync(0xffffffffu, x, 16);
        const int r = nq * 8 + 2 * t + e;
        if (g == 0) {
          sh_m[warp][r] = m[nq][e];
          sh_l[warp][r] = x;
        }
        // dims 16 g' .. of row r: tile k holds dims D/8 g + 2k and + 2k + 1
        float* dst = sh_o + warp * kWarpFloats + r * D + order<D>(g) * (D / 8);
#pragma unroll
        for (int k = 0; k < MT; k += 2)
          *reinterpret_cast<float4*>(dst + 2 * k) =
              make_float4(value(o[nq][k][e]), value(o[nq][k][e + 2]), value(o[nq][k + 1][e]), value(o[nq][k + 1][e + 2]));
      }
    __syncthreads();
    const bool whole = ta == 0 && tb == tiles;
    const int part = ta > 0 ? 0 : 1;
    float* po = p.part_o + ((int64_t)w.index * 2 + part) * kAttendRows * D;
    float2* pml = p.part_ml + ((int64_t)w.index * 2 + part) * kAttendRows;
    const int live = min(rows, R);
    for (int e = threadIdx.x; e < live * D / 4; e += kThreads) {
      const int r = e / (D / 4), d = e % (D / 4) * 4;
      float mx = -INFINITY;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) mx = fmaxf(mx, sh_m[k][r]);
      const float ref = mx == -INFINITY ? 0.f : mx;
      float sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kWarps; ++k) {
        const float f = fast_exp2(sh_m[k][r] - ref);
        const float4 x = *reinterpret_cast<const float4*>(sh_o + k * kWarpFloats + r * D + d);
        sum = fmaf(sh_l[k][r], f, sum);
        v[0] = fmaf(x.x, f, v[0]);
        v[1] = fmaf(x.y, f, v[1]);
        v[2] = fmaf(x.z, f, v[2]);
        v[3] = fmaf(x.w, f, v[3]);
      }
      const int row = rt * R + r, j = div_group(p, row);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (nan_first[d + q] < (p.causal ? s.len - s.rows + j + 1 : s.len)) v[q] = __int_as_float(0x7fc00000);
      if (!in_bounds(s.row0 + j < p.total_rows && h * p.G + row - j * p.G < p.H, p.c.status, kSiteAttendRow)) continue;
      if (whole) {
        const int64_t to = (s.row0 + j) * p.H + h * p.G + row - j * p.G;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        uint16_t o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = out_bits(sum == 0.f ? 0.f : v[q] * inv, p.bf16);
        *reinterpret_cast<uint2*>(p.out + to * D + d) = make_uint2(o[0] | ((uint32_t)o[1] << 16), o[2] | ((uint32_t)o[3] << 16));
        if (d == 0 && p.lse) p.lse[to] = sum == 0.f ? -INFINITY : (mx + log2f(sum)) * 0.69314718056f;
      } else {
        *reinterpret_cast<float4*>(po + r * D + d) = make_float4(v[0], v[1], v[2], v[3]);
        if (d == 0) pml[r] = make_float2(mx, sum);
      }
    }
    if (!whole) {
      __syncthreads();
      const int2 who = item_stretches<kOver>(line, x0);
      const int first = who.x, last = who.y;
      const bool fits = in_bounds(first >= 0 && first < last && last < line.stretches && line.stretches <= kAttendCtas &&
                                      w.index >= first && w.index <= last, p.c.status, kSiteAttendPart);
      if (threadIdx.x == 0) sh_last = fits && arrive_count(&p.counters[first]) == last - first;
      __syncthreads();
      if (sh_last) {
        if (threadIdx.x == 0) p.counters[first] = 0;
        // Weights of the parts (a warp a row, a lane a part), then the sums, all of a
        // block's parts in flight; the partial sums of this CTA's warps are done with.
        constexpr int kBlock = 256;
        float* wt = sh_o;  // [R][kBlock]
        for (int c0 = first; c0 <= last; c0 += kBlock) {
          const int n = min(last - c0 + 1, kBlock);
          for (int r = warp; r < live; r += kWarps) {
            auto ml = [&](int c) { return __ldcg(&p.part_ml[((int64_t)c * 2 + (c == first ? 1 : 0)) * kAttendRows + r]); };
            float mx = -INFINITY, sum = 0.f;
            for (int c = first + lane; c <= last; c += 32) mx = fmaxf(mx, ml(c).x);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float ref = mx == -INFINITY ? 0.f : mx;
            for (int c = first + lane; c <= last; c += 32) {
              const float2 x = ml(c);
              const float f = fast_exp2(x.x - ref);
              sum += x.y * f;
              if (c >= c0 && c < c0 + n) wt[r * kBlock + c - c0] = f;
            }
            sum = warp_sum(sum);
            if (lane == 0) {
              sh_m[0][r] = mx;
              sh_l[0][r] = sum;
            }
          }
          __syncthreads();
          for (int e = threadIdx.x; e < live * D / 4; e += kThreads) {
            const int r = e / (D / 4), d = e % (D / 4) * 4;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            float4* keep = reinterpret_cast<float4*>(p.part_o + (((int64_t)first * 2 + 1) * kAttendRows + r) * D + d);
#pragma unroll 4
            for (int k = 0; k < n; ++k) {
              const int c = c0 + k;
              const float4 x = __ldcg(reinterpret_cast<const float4*>(
                  p.part_o + (((int64_t)c * 2 + (c == first ? 1 : 0)) * kAttendRows + r) * D + d));
              const float f = wt[r * kBlock + k];
              acc.x = fmaf(x.x, f, acc.x);
              acc.y = fmaf(x.y, f, acc.y);
              acc.z = fmaf(x.z, f, acc.z);
              acc.w = fmaf(x.w, f, acc.w);
            }
            if (c0 > first) {  // the blocks before, kept in the first part's place
              const float4 x = *keep;
              acc = make_float4(acc.x + x.x, acc.y + x.y, acc.z + x.z, acc.w + x.w);
            }
            if (c0 + n <= last) {
              *keep = acc;
            } else {
              const float sum = sh_l[0][r], mx = sh_m[0][r], inv = sum == 0.f ? 0.f : 1.f / sum;
              const int row = rt * R + r, j = div_group(p, row);
              const int64_t to = (s.row0 + j) * p.H + h * p.G + row - j * p.G;
              if (!in_bounds(to < p.total_rows * p.H, p.c.status, kSiteAttendRow)) continue;
              const float v[4] = {acc.x, acc.y, acc.z, acc.w};
              uint16_t o[4];
#pragma unroll
              for (int q = 0; q < 4; ++q) o[q] = out_bits(sum == 0.f ? 0.f : v[q] * inv, p.bf16);
              *reinterpret_cast<uint2*>(p.out + to * D + d) =
                  make_uint2(o[0] | ((uint32_t)o[1] << 16), o[2] | ((uint32_t)o[3] << 16));
              if (d == 0 && p.lse) p.lse[to] = sum == 0.f ? -INFINITY : (mx + log2f(sum)) * 0.69314718056f;
            }
          }
          __syncthreads();
        }
      }
    }
    if (TMA) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the next copies come by another proxy
    __syncthreads();  // the shared results are free again
    // (the next segment has the other notes: its first warp may be there before the last one clears these)
    for (int d = threadIdx.x; d < D; d += kThreads) nan_first[d] = 0x7fffffff;
    nan_first = nan_first == sh_nan[0] ? sh_nan[1] : sh_nan[0];
  } while (walk_next<R, kTile, kOver>(p, w, x0));
}

template <int D, int NQ, bool TMA>
int launch(const AttendParams& p, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t st) {
  constexpr int smem = kWarps * 4 * kTile * D + 1024;
  static std::atomic<uint64_t> ready{0};  // devices whose shared memory limit is raised
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return OCCAM_ERR_CUDA;
  if (!((ready.load(std::memory_order_acquire) >> dev) & 1)) {
    if (cudaFuncSetAttribute(attend_rows_kernel<D, NQ, TMA>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
      return OCCAM_ERR_CUDA;
    ready.fetch_or(uint64_t(1) << dev, std::memory_order_release);
  }
  const int grid = std::min(cache_sms() * (NQ == 1 ? 3 : 2), kAttendCtas);
  return launch_after(attend_rows_kernel<D, NQ, TMA>, dim3((unsigned)grid), kThreads, smem, st, p, mk, mv) &&
                 cudaGetLastError() == cudaSuccess
             ? OCCAM_OK
             : OCCAM_ERR_CUDA;
}

template <int D, int NQ>
int launch_rows(const AttendParams& p, cudaStream_t st) {
  CUtensorMap mk{}, mv{};
  // Tensor copies where every row of a tile is wanted; with keep flags, rows
  // one by one (a hidden row is not read). 64 single tokens over 2,300, of which 10 % are seen: 83 us,
  // by tensor copies 94; half 93 and 92; 90 % 94.5 and 92; without flags 65.
  if (p.keep) return launch<D, NQ, false>(p, mk, mv, st);
  const int box = std::min(p.c.T, kTile);
  if (!encode_blocks(&mk, p.c, p.c.k, D, box, true) || !encode_blocks(&mv, p.c, p.c.v, D, box, true)) return OCCAM_ERR_CUDA;
  return launch<D, NQ, true>(p, mk, mv, st);
}

}  // namespace

bool occam::encode_blocks(CUtensorMap* m, const CacheDev& c, const void* codes, int dim, int box_rows, bool swizzle) {
  static const PFN_cuTensorMapEncodeTiled_v12000 enc = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool found = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) ==
                           cudaSuccess && q == cudaDriverEntryPointSuccess;
    return found ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f) : nullptr;
  }();
  if (!enc) return false;
  const cuuint64_t rows = (cuuint64_t)c.heads * c.T;
  cuuint64_t gdim[3] = {(cuuint64_t)dim, rows, (cuuint64_t)c.layers * c.pages};
  cuuint64_t gstride[2] = {(cuuint64_t)dim, rows * dim};
  cuuint32_t box[3] = {(cuuint32_t)dim, (cuuint32_t)box_rows, 1};
  cuuint32_t es[3] = {1, 1, 1};
  const CUtensorMapSwizzle sw =
      !swizzle ? CU_TENSOR_MAP_SWIZZLE_NONE : dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(codes), gdim, gstride, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

#define OCCAM_TRY(x)                 \
  do {                               \
    int _rc = (x);                   \
    if (_rc != OCCAM_OK) return _rc; \
  } while (0)

extern "C" int occam_cache_attend(const occam_cache* cache, const occam_attend_args* a, void* workspace,
                                  size_t workspace_bytes, occam_stream_t stream) {
  const NvtxRange nvtx("occam_cache_attend");
  launch_counter() = 0;
  OCCAM_TRY(check_cache(cache));
  if (!a) return OCCAM_ERR_INVALID_ARG;
  if (a->dtype != OCCAM_BF16 && a->dtype != OCCAM_F16) return OCCAM_ERR_UNSUPPORTED;
  if (a->layer < 0 || a->layer >= cache->layers || a->total_rows < 0 || a->total_rows > 0x7fffffff || a->n < 0 ||
      a->n > cache->max_seqs || a->max_rows < 0 || a->heads < 1 || a->heads % cache->heads != 0 || !(a->scale >= 0.f) ||
      !(a->scale < INFINITY))
    return OCCAM_ERR_INVALID_ARG;
  const int G = a->heads / cache->heads;
  if (G > 64 || a->total_rows * G > 0x7fffffff) return OCCAM_ERR_UNSUPPORTED;
  if (a->keep && (!a->keep_off || a->total_keep < 0)) return OCCAM_ERR_INVALID_ARG;
  CacheWs w;
  OCCAM_TRY(check_cache_ws(cache, 0, workspace, workspace_bytes, &w));
  if (a->n == 0 || a->total_rows == 0) return OCCAM_OK;
  if (!a->q || !a->out || !a->seqs || !a->row_off || !aligned16(a->q) || !aligned16(a->out) || (a->q_row & 7) ||
      a->q_row < (int64_t)a->heads * cache->dim)
    return OCCAM_ERR_INVALID_ARG;
  AttendParams p{};
  p.c = cache_dev(cache, workspace, w);
  p.layer = a->layer;
  p.n = a->n;
  p.H = a->heads;
  p.G = G;
  // ceil(2^(31 + s) / G) with 2^s >= G: exact for 31-bit numbers
  uint32_t sh = 0;
  while ((1 << sh) < G) ++sh;
  p.g_shift = 31 + sh;
  p.g_mul = (uint32_t)(((uint64_t(1) << p.g_shift) + G - 1) / G);
  p.causal = a->causal ? 1 : 0;
  p.bf16 = a->dtype == OCCAM_BF16;
  p.row_lo = 0;
  p.row_hi = 0x7fffffff;
  p.total_rows = a->total_rows;
  p.q_row = a->q_row;
  p.total_keep = a->total_keep;
  p.q = static_cast<const uint16_t*>(a->q);
  p.out = static_cast<uint16_t*>(a->out);
  p.lse = a->lse;
  p.seqs = a->seqs;
  p.row_off = a->row_off;
  p.keep = a->keep;
  p.keep_off = a->keep_off;
  const double scale = a->scale > 0.f ? (double)a->scale : 1.0 / std::sqrt((double)cache->dim);
  p.scale_log2 = (float)(scale * 1.4426950408889634);
  p.counters = ws_at<int32_t>(workspace, w.counters);
  p.part_o = ws_at<float>(workspace, w.part_o);
  p.part_ml = ws_at<float2>(workspace, w.part_ml);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  // Sequences with more than kFewRows query rows a key head go to the
  // tensor-core kernel, the others are this file's; one launch where the rows allow only one of them.
  const int64_t most = (int64_t)a->max_rows * G;
  if (most > kFewRows) {
    p.row_lo = a->n == 1 ? 0 : kFewRows;
    OCCAM_TRY(launch_attend_tc(p, cache->dim, st));
    if (a->n == 1) return OCCAM_OK;  // whatever its rows are
    p.row_lo = 0;
    p.row_hi = kFewRows;
  }
  // One column tile where no sequence has more than 8 rows. (Which rows are left for this launch is
  // only known on the device: 63 single tokens beside a prefix of 2,000 take two column tiles, 174 us in all
  // where one would give 154; but 64 x 16 rows take 98 us with two and 116 with one.)
  const bool few = most <= 8;
  if (cache->dim == 128) return few ? launch_rows<128, 1>(p, st) : launch_rows<128, 2>(p, st);
  return few ? launch_rows<64, 1>(p, st) : launch_rows<64, 2>(p, st);
}
