// prompt.cu -- attention of whole prompts (packed sequences of 16-bit rows with
// grouped heads) on the fifth-generation tensor cores, and the C-ABI entry.
//
// One pass over the keys: with s_k = scale q.k in log2 units and a reference m of
// the row, l = sum 2^(s_k - m), O = sum 2^(s_k - m) v_k; both are rescaled only where
// the maximum grew by more than 2^8 since the last reference. 4 D operations and one exponential
// a (row, head, key).
// An item is 256 rows: two tiles of 128, each 128 / P tokens x P heads of one key head's group
// (P: the group's largest power of two, so that grouped heads read their keys
// once and a causal tile spans few tokens). One CTA an SM takes items from a counter; 16 warps in six roles
// that run through the items one after the other without a barrier between them:
//  - warp 13 copies queries, keys and values to shared memory (TMA);
//  - warps 12 and 14 issue the products of a row tile each: S = Q K^T into tensor memory, 64 keys at a
//    time, O += P V with P read from tensor memory. While one half of the scores is in the
//    softmax, the other is multiplied; the next item's scores follow the last product of the one before;
//  - warps 0-3 and 4-7 hold a row a thread: scores, maximum, exponentials, P back as 16 bits;
//  - warps 8-11 write the results: O from tensor memory over shared memory as whole rows;
//  - warp 15 takes items and tells the others of them; it looks values over that some row does not see: rows past the sequence's
//    end become zeros, and so do values that are not finite, which are noted and put back into
//    the results of the rows that see them.
// P is rounded to the type of the values (both operands of a product have one type), l sums the unrounded P.
// Bound at 128 dims by the products: 8,257 causal rows of 32 heads in 353 us, 1,580 TFLOP/s (0.84 of cuBLAS' measured rate),
// 378 us where every pass has other inputs;
// at 64 to 80 by the softmax's chain (scores, maximum, exponentials, P; two warps a scheduler do not hide its
// latencies): 27 k full rows (12 images) of 16 heads of 72 in 370 us, tensor pipe 48 % busy, issue 48 %, exponentials 38 %. Many short prompts
// (64 of about 310, 32 key heads) are bound by HBM: 154 us, 0.65 of a plain copy.
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "nvtx.cuh"
#include "prompt.cuh"

using namespace occam;

namespace {

constexpr int kThreads = 512;
constexpr int kK = 128;          // keys of a tile
constexpr int kItems = 3;        // items known ahead
constexpr int kBlock = 128 * 128;  // bytes of 128 rows x 64 dims
constexpr int kRegSoftmax = 168, kRegWrite = 88, kRegIssue = 88;  // 2 x 168 + 88 + 88 = 4 x 128
constexpr float kLazy = 8.f;     // log2 growth of a maximum before O is rescaled
constexpr int kNever = 0x7fffffff;

template <int DP>
struct Shape {
  static constexpr int kBlocks = DP > 64 ? 2 : 1;     // blocks of 64 dims
  static constexpr int kTile = kBlocks * kBlock;      // bytes of a tile of 128 rows
  static constexpr int kStages = DP > 64 ? 2 : 4;
  static constexpr int kKSteps = DP / 16;
};

template <int STAGES>
struct Shared {
  uint64_t q_full[2], q_free[2], k_full[STAGES], k_free[STAGES], v_full[STAGES], v_ready[STAGES], v_free[STAGES], s_full[2][2],
      p_full[2][2], o_done[2][2], o_full[2], o_free[2], inv_full[2], inv_free[2], item_full[kItems], item_free[kItems], drain;
  PromptItem item[kItems];
  uint32_t tmem;
  int stop;
  float inv[2][128];
  // of each item: the first key whose value is NaN, +inf, -inf in a dim, among those taken out
  int odd[kItems];
  int first[kItems][3][128];
  PromptList list;
};

// items of a sequence, and the item at a place: blocks of rows from the last to the first, heads inner
struct Count {
  const PromptParams& p;
  __device__ __forceinline__ int operator()(const PromptSeq& s) const {
    const int per = 256 >> p.log2P;
    return (s.rows / per + (s.rows % per != 0)) * (p.H >> p.log2P);
  }
};
__device__ __forceinline__ int key_steps(const PromptParams& p, const PromptSeq& s, int tok_last) {
  const int lim = min(prompt_limit(p, s.rows, s.keys, tok_last), s.keys);
  return max((lim + kK - 1) / kK, 1);  // (where nothing is seen, one tile of hidden keys gives the rows their zeros)
}

// Steps whose keys every row of the item sees
__device__ __forceinline__ int whole_steps(const PromptParams& p, const PromptItem& x) {
  return min(prompt_limit(p, x.rows, x.keys, (x.tile * 2) << (7 - p.log2P)), x.keys) / kK;
}

#define WAIT(bar, parity) PROMPT_WAIT(bar, parity)

template <int DP, class Sh>
__device__ __forceinline__ void load_role(const PromptParams& p, Sh& sh, const CUtensorMap& map_q, const CUtensorMap& map_k,
                                          const CUtensorMap& map_v, unsigned char* q_smem, unsigned char* k_smem, unsigned char* v_smem) {
  using S = Shape<DP>;
  const int lane = threadIdx.x & 31;
  uint32_t j = 0, nq[2] = {0, 0};
  for (uint32_t i = 0;; ++i) {
    WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
    const PromptItem it = sh.item[i % kItems];
    if (it.steps == 0) return;
    const int tt = 128 >> p.log2P, head = it.hb << p.log2P, kv = head / p.G;
    for (int k = 0; k < it.steps; ++k, ++j) {
      const int st = j % S::kStages;
      const uint32_t turn = ((j / S::kStages) & 1) ^ 1;
      const int key = (int)(it.key0 + (int64_t)k * kK);
      WAIT(sh.k_free[st], turn);
      if (lane == 0) {
        tc::bar_expect_tx(&sh.k_full[st], S::kTile);
        for (int b = 0; b < S::kBlocks; ++b) tc::tma_load_3d(k_smem + st * S::kTile + b * kBlock, &map_k, b * 64, kv, key, &sh.k_full[st]);
      }
      if (k == 0) {
        for (int t = 0; t < 2; ++t) {
          if (it.nk[t] == 0) continue;
          WAIT(sh.q_free[t], (nq[t] & 1) ^ 1);
          ++nq[t];
          if (lane == 0) {
            const int row = (int)(it.row0 + (int64_t)(it.tile * 2 + t) * tt);
            tc::bar_expect_tx(&sh.q_full[t], S::kTile);
            for (int b = 0; b < S::kBlocks; ++b)
              tc::tma_load_3d(q_smem + t * S::kTile + b * kBlock, &map_q, b * 64, head, row, &sh.q_full[t]);
          }
        }
      }
      WAIT(sh.v_free[st], turn);
      if (lane == 0) {
        tc::bar_expect_tx(&sh.v_full[st], S::kTile);
        for (int b = 0; b < S::kBlocks; ++b) tc::tma_load_3d(v_smem + st * S::kTile + b * kBlock, &map_v, b * 64, kv, key, &sh.v_full[st]);
      }
      __syncwarp();
    }
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
    __syncwarp();
  }
}

// ---------------------------------------------------------------- issuing
// Row tile t. Step by step and half by half: O += P V of the step before, then S of this step in the place
// of that P. One lane does it all: a turn of the whole warp with an election for every group of products took longer than
// the products. (A descriptor's address field counts 16 bytes.)
template <int DP, bool BF16, class Sh>
__device__ __forceinline__ void issue_role(const PromptParams& p, Sh& sh, uint32_t q_smem, uint32_t k_smem, uint32_t v_smem,
                                           uint32_t tmem, int t) {
  using S = Shape<DP>;
  constexpr uint32_t id_s = tc::idesc16(BF16, 128, 64, false), id_o = tc::idesc16(BF16, 128, DP, true);
  const uint64_t kmajor = tc::sdesc_sw128(0), mnmajor = tc::sdesc_mn_sw128(0, kBlock);
  const uint32_t km = tc::desc_hi(kmajor), mn = tc::desc_hi(mnmajor);
  const uint32_t dq = (uint32_t)kmajor + ((q_smem + t * S::kTile) >> 4), dk = (uint32_t)kmajor + (k_smem >> 4),
                 dv = (uint32_t)mnmajor + (v_smem >> 4);
  const uint32_t o_at = tmem + 256 + t * 128, s_at = tmem + t * 128;
  uint32_t j = 0, products = 0;  // steps; this row tile's steps whose product was issued
  uint32_t n_q = 0, n_o = 0;     // this row tile's items whose scores, whose products have begun
  uint32_t looked = 0;           // a bit a stage: how often (mod 2) its values were looked at
  struct {
    bool any, mine, first, last, look;
  } was = {false, false, false, false, false};
  uint32_t i = 0;
  int k = 0, steps = 0, nk = 0, whole = 0;  // whole: steps whose keys every row of the item sees
  for (;;) {
    if (k == steps) {
      if (i > 0) tc::bar_arrive(&sh.item_free[(i - 1) % kItems]);
      WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
      const PromptItem& x = sh.item[i % kItems];
      steps = x.steps;
      nk = x.nk[t];
      whole = whole_steps(p, x);
      k = 0;
      ++i;
    }
    const bool end = steps == 0, mine = !end && k < nk;
    const uint32_t st = j % S::kStages, before = (j - 1) % S::kStages;
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
      if (was.any) {
        if (h == 0) {
          WAIT(sh.v_full[before], ((j - 1) / S::kStages) & 1);
          if (was.look) {
            WAIT(sh.v_ready[before], (looked >> before) & 1);
            looked ^= 1u << before;
          }
        }
        if (was.mine) {
          if (h == 0 && was.first) {
            WAIT(sh.o_free[t], (n_o & 1) ^ 1);
            ++n_o;
          }
          WAIT(sh.p_full[t][h], products & 1);
          tc::fence_after();
          {
            const uint32_t vd = dv + before * (S::kTile >> 4) + h * (64 * 128 >> 4);
#pragma unroll
            for (int q = 0; q < 4; ++q)
              tc::mma16_ts(o_at, s_at + h * 64 + q * 8, vd + q * (2048 >> 4), mn, id_o, q > 0 || h > 0 || !was.first);
            tc::mma_commit(&sh.o_done[t][h]);
            if (h == 1 && was.last) tc::mma_commit(&sh.o_full[t]);
          }
        }
      }
      if (mine) {
        if (h == 0) {
          if (k == 0) {
            WAIT(sh.q_full[t], n_q & 1);
            ++n_q;
          }
          WAIT(sh.k_full[st], (j / S::kStages) & 1);
          tc::fence_after();
        }
        {
          const uint32_t kd = dk + st * (S::kTile >> 4) + h * (64 * 128 >> 4);
#pragma unroll
          for (int q = 0; q < S::kKSteps; ++q) {
            const int o = (q >> 2) * (kBlock >> 4) + (q & 3) * 2;
            tc::mma16_ss(s_at + h * 64, dq + o, km, kd + o, km, id_s, q > 0);
          }
          tc::mma_commit(&sh.s_full[t][h]);
        }
      }
    }
    if (!end && !mine) WAIT(sh.k_full[st], (j / S::kStages) & 1);  // (a stage is given back after it was filled)
    // (without products of its own the warp just arrives)
    {
      if (was.any) was.mine ? tc::mma_commit(&sh.v_free[before]) : tc::bar_arrive(&sh.v_free[before]);
      if (!end) mine ? tc::mma_commit(&sh.k_free[st]) : tc::bar_arrive(&sh.k_free[st]);
      if (mine && k == nk - 1) tc::mma_commit(&sh.q_free[t]);
    }
    if (was.mine) ++products;
    if (end) return;
    was.any = true;
    was.mine = mine;
    was.first = k == 0;
    was.last = k == nk - 1;
    was.look = k >= whole;
    ++j;
    ++k;
  }
}

// ---------------------------------------------------------------- a row a thread
template <int DP, bool BF16, class Sh>
__device__ __forceinline__ void softmax_role(const PromptParams& p, Sh& sh, uint32_t tmem, int t) {
  // P of f16 values is held 2^7 times as large: at most 2^15 (f16 ends at 2^16), and what is 2^-21 of a row's
  // reference still has f16's 11 bits. bf16 has fp32's range: P is held 2^-16 times as large, at most 2^-8, so that sums
  // of values near bf16's end stay finite (those of 65,536 keys, 256 where a reference lags as far as it may) and
  // values down to 2^-110 keep their bits.
  constexpr float kLift = BF16 ? -16.f : 7.f;
  const int r = threadIdx.x & 127, lane = threadIdx.x & 31;
  const uint32_t lanes = (uint32_t)(r & ~31) << 16;
  const uint32_t s_at = tmem + t * 128 + lanes, o_at = tmem + 256 + t * 128 + lanes;
  const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
  uint32_t it = 0, n = 0;  // halves, items of this row tile
  for (uint32_t i = 0;; ++i) {
    WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
    const PromptItem& x = sh.item[i % kItems];
    const int steps = x.steps, nk = x.nk[t], rows = x.rows, keys = x.keys;
    if (steps == 0) return;
    const int first = (x.tile * 2 + t) << (7 - p.log2P), tok = first + (r >> p.log2P);
    const int64_t at = (x.row0 + tok) * p.H + (x.hb << p.log2P) + (r & ((1 << p.log2P) - 1));
    __syncwarp();
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
    if (nk == 0) continue;
    const int limit = min(prompt_limit(p, rows, keys, tok), keys), common = min(prompt_limit(p, rows, keys, first), keys);
    float ref = -INFINITY, l = 0.f;
    float top = -INFINITY;  // of the raw scores
#pragma unroll 1
    for (int k = 0; k < 2 * nk; ++k, ++it) {
      const int h = k & 1, key0 = k * 64;
      WAIT(sh.s_full[t][h], (it >> 1) & 1);
      tc::fence_after();
      uint32_t v[64];
      tc::tmem_ld64(s_at + 64 * h, v);
      tc::wait_ld64(v);
      if (PROMPT_RARE(key0 + 64 > common)) {
        const int lim = limit - key0;
#pragma unroll
        for (int e = 0; e < 64; ++e) v[e] = e < lim ? v[e] : 0xff800000u;
      }
      float m0 = top, m1 = -INFINITY, m2 = -INFINITY, m3 = -INFINITY;
#pragma unroll
      for (int e = 0; e < 64; e += 8) {
        m0 = tc::fmax3(m0, __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
        m1 = tc::fmax3(m1, __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]));
        m2 = tc::fmax3(m2, __uint_as_float(v[e + 4]), __uint_as_float(v[e + 5]));
        m3 = tc::fmax3(m3, __uint_as_float(v[e + 6]), __uint_as_float(v[e + 7]));
      }
      top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
      const float m = top * p.scale_log2;
      bool move = false;
      float fall = 1.f;
      if (m > ref + kLazy || ref == -INFINITY) {
        if (m != ref) {
          fall = ref == -INFINITY ? 0.f : fast_exp2(ref - m);
          l *= fall;
          move = true;
          ref = m;
        }
      }
      // O in units of the new reference (nothing is there before the first product)
      if (PROMPT_RARE(k > 0 && __any_sync(0xffffffffu, move))) {
        // the product of the half before (the one before that is done: these scores came after it)
        WAIT(sh.o_done[t][h ^ 1], ((it - 1) >> 1) & 1);
        tc::fence_after();
#pragma unroll 1
        for (int c = 0; c < DP / 16; ++c) {
          uint32_t o[16];
          tc::tmem_ld16(o_at + 16 * c, o);
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * fall);
          tc::tmem_st16(o_at + 16 * c, o);
        }
      }
      const float add = kLift - (ref == -INFINITY ? 0.f : ref);
      const float2 add2 = make_float2(add, add);
      float2 sum = make_float2(0.f, 0.f);
      uint32_t pk[32];
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        float2 y = tc::fma2(make_float2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), scale2, add2);
        y.x = fast_exp2(y.x);
        y.y = fast_exp2(y.y);
        sum = tc::add2(sum, y);
        pk[e] = pack16<BF16>(y.x, y.y);
      }
      l += sum.x + sum.y;
      tc::tmem_st32(s_at + 64 * h, pk);  // (over scores that are in registers already)
      tc::tmem_wait_st();
      tc::fence_before();
      tc::bar_arrive(&sh.p_full[t][h]);
    }
    WAIT(sh.inv_free[t], (n & 1) ^ 1);
    sh.inv[t][r] = l == 0.f ? 0.f : 1.f / l;
    tc::bar_arrive(&sh.inv_full[t]);
    ++n;
    if (p.lse && tok < rows && in_bounds(at < p.total_rows * p.H, p.status, kSitePromptRow))
      p.lse[at] = l == 0.f ? -INFINITY : (BF16 ? ref + log2f(l * 65536.f) : ref + log2f(l) - kLift) * 0.69314718056f;
  }
}

// ---------------------------------------------------------------- results
template <bool BF16>
__device__ __forceinline__ float value16(uint16_t x) {
  return BF16 ? __uint_as_float((uint32_t)x << 16) : __half2float(__ushort_as_half(x));
}
template <int DP, bool BF16, class Sh>
__device__ __forceinline__ void write_role(const PromptParams& p, Sh& sh, unsigned char* stage_all, uint32_t tmem) {
  const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, r = warp * 32 + lane;
  const uint32_t lanes = (uint32_t)(warp * 32) << 16;
  unsigned char* stage = stage_all + warp * (32 * 128);
  uint32_t n[2] = {0, 0};
  for (uint32_t i = 0;; ++i) {
    WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
    const PromptItem x = sh.item[i % kItems];
    if (x.steps == 0) return;
    const int pieces = p.dim / 8;
    auto row_at = [&](int t, int rr, bool& there) {
      const int tok = ((x.tile * 2 + t) << (7 - p.log2P)) + (rr >> p.log2P);
      there = tok < x.rows;
      return ((x.row0 + tok) * p.H + (x.hb << p.log2P) + (rr & ((1 << p.log2P) - 1)));
    };
#pragma unroll 1
    for (int t = 0; t < 2; ++t) {
      if (x.nk[t] == 0) continue;
      WAIT(sh.inv_full[t], n[t] & 1);
      const float inv = sh.inv[t][r];
      tc::bar_arrive(&sh.inv_free[t]);
      WAIT(sh.o_full[t], n[t] & 1);
      tc::fence_after();
      ++n[t];
      // Blocks of 64 dims go through shared memory one after the other; the second one waits in registers, so that
      // the tensor memory is free for the next item before anything is written.
      auto read16 = [&](int c, uint32_t* w) {
        uint32_t o[16];
        tc::tmem_ld16(tmem + 256 + t * 128 + lanes + c, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x0 = __uint_as_float(o[2 * e]) * inv, x1 = __uint_as_float(o[2 * e + 1]) * inv;
          w[e] = pack16<BF16>(inv == 0.f ? 0.f : x0, inv == 0.f ? 0.f : x1);
        }
      };
      auto put16 = [&](int c, const uint32_t* w) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
          *reinterpret_cast<uint4*>(stage + lane * 128 + (((c / 8 + e) ^ (lane & 7)) << 4)) =
              make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
      };
      auto flush = [&](int b) {
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int rr = e * 4 + lane / 8, c = lane % 8;
          bool there;
          const int64_t at = row_at(t, warp * 32 + rr, there);
          const uint4 v = *reinterpret_cast<const uint4*>(stage + rr * 128 + ((c ^ (rr & 7)) << 4));
          if (there && b * 8 + c < pieces && in_bounds(at < p.total_rows * p.H, p.status, kSitePromptRow))
            *reinterpret_cast<uint4*>(p.out + at * p.dim + b * 64 + c * 8) = v;
        }
        __syncwarp();
      };
      constexpr int kRest = DP > 64 ? DP - 64 : 0;
      uint32_t rest[kRest / 2 + 8];
#pragma unroll
      for (int c = 0; c < DP - kRest; c += 16) {
        uint32_t w[8];
        read16(c, w);
        put16(c, w);
      }
#pragma unroll
      for (int c = 0; c < kRest; c += 16) read16(64 + c, rest + c / 2);
      tc::fence_before();
      tc::bar_arrive(&sh.o_free[t]);
      flush(0);
      if (kRest) {
#pragma unroll
        for (int c = 0; c < kRest; c += 16) put16(c, rest + c / 2);
        flush(1);
      }
      if (PROMPT_RARE(*reinterpret_cast<volatile int*>(&sh.odd[i % kItems]))) {
        // values that are not finite and were taken out of the product, for the rows that see them
        bool there;
        const int64_t at = row_at(t, r, there);
        const int tok = ((x.tile * 2 + t) << (7 - p.log2P)) + (r >> p.log2P);
        const int limit = min(prompt_limit(p, x.rows, x.keys, tok), x.keys);
        const int* first = sh.first[i % kItems][0];
        if (there && in_bounds(at < p.total_rows * p.H, p.status, kSitePromptRow)) {
#pragma unroll 1
          for (int d = 0; d < p.dim; ++d) {
            float y = first[d] < limit ? NAN : 0.f;
            if (first[128 + d] < limit) y += INFINITY;
            if (first[256 + d] < limit) y -= INFINITY;
            uint16_t* to = p.out + at * p.dim + d;
            if (y != 0.f) *to = (uint16_t)pack16<BF16>(value16<BF16>(*to) + y, 0.f);
          }
        }
      }
    }
    __syncwarp();
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
  }
}

// ---------------------------------------------------------------- values that some row does not see
// sum += 0 x, two values a word
template <bool BF16>
__device__ __forceinline__ void add_zero_times(uint32_t& sum, uint32_t x) {
  if (BF16)
    asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(x), "r"(0));
  else
    asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(x), "r"(0));
}
template <int DP, bool BF16, class Sh>
__device__ __forceinline__ void look_role(const PromptParams& p, Sh& sh, unsigned char* v_smem) {
  using S = Shape<DP>;
  const int lane = threadIdx.x & 31;
  PromptTaker taker;
  uint32_t told = 0;
  auto tell = [&]() -> bool {
    PromptItem& it = sh.item[told % kItems];
    if (!prompt_wait(&sh.item_free[told % kItems], ((told / kItems) & 1) ^ 1, &sh.stop)) return false;
    if (sh.odd[told % kItems]) {  // the notes of the item that was here (every role is done with it)
      for (int d = lane; d < 3 * 128; d += 32) sh.first[told % kItems][0][d] = kNever;
      __syncwarp();
      if (lane == 0) sh.odd[told % kItems] = 0;
    }
    const int place = taker.take(p, sh.list, Count{p});
    const PromptSeq& s = taker.s;
    if (place >= 0) {
      const int hbs = p.H >> p.log2P, log_tt = 7 - p.log2P, per = 2 << log_tt;
      const int blocks = (s.rows + per - 1) / per;
      const int tile = blocks - 1 - place / hbs, hb = place % hbs, tok0 = tile * per;
      const int left = s.rows - tok0;
      const int nk0 = key_steps(p, s, tok0 + min(left, 1 << log_tt) - 1);
      const int nk1 = left > (1 << log_tt) ? key_steps(p, s, tok0 + min(left, per) - 1) : 0;
      if (lane == 0) {
        it.row0 = s.row0;
        it.key0 = s.key0;
        it.rows = s.rows;
        it.keys = s.keys;
        it.tile = tile;
        it.hb = hb;
        it.steps = max(nk0, nk1);
        it.nk[0] = nk0;
        it.nk[1] = nk1;
      }
    } else if (lane == 0) {
      it.steps = 0;
    }
    __syncwarp();
    if (lane == 0) tc::bar_arrive(&sh.item_full[told % kItems]);
    __syncwarp();
    ++told;
    return true;
  };
  if (!tell()) return;
  uint32_t j = 0;
  for (uint32_t i = 0;; ++i) {
    WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
    const PromptItem x = sh.item[i % kItems];
    if (x.steps == 0) return;
    if (!tell()) return;  // the next one, while the first copies are under way
    const int whole = whole_steps(p, x);
#pragma unroll 1
    for (int k = 0; k < x.steps; ++k, ++j) {
      const int st = j % S::kStages;
      WAIT(sh.v_full[st], (j / S::kStages) & 1);
      if (k >= whole) {
        unsigned char* v = v_smem + st * S::kTile;
        const int live = min(max(x.keys - k * kK, 0), kK);
        // x 0 is 0 but for infinities and NaN, whose NaN stays in the sum
        uint32_t sum[4] = {0, 0, 0, 0};
#pragma unroll 1
        for (int b = 0; b < S::kBlocks; ++b) {
          uint4* piece = reinterpret_cast<uint4*>(v + b * kBlock);
          // four rows a turn, a piece of 8 values a lane (pieces past the dims hold zeros)
#pragma unroll 8
          for (int e = lane; e < live * 8; e += 32) {
            const uint4 w = piece[e];
            add_zero_times<BF16>(sum[0], w.x);
            add_zero_times<BF16>(sum[1], w.y);
            add_zero_times<BF16>(sum[2], w.z);
            add_zero_times<BF16>(sum[3], w.w);
          }
#pragma unroll 4
          for (int e = live * 8 + lane; e < kK * 8; e += 32) piece[e] = make_uint4(0, 0, 0, 0);
        }
        const bool hit = ((sum[0] | sum[1] | sum[2] | sum[3]) & 0x7fff7fffu) != 0;
        if (PROMPT_RARE(__any_sync(0xffffffffu, hit))) {
          if (lane == 0) *reinterpret_cast<volatile int*>(&sh.odd[i % kItems]) = 1;
#pragma unroll 1
          for (int e = lane; e < S::kBlocks * live * 8; e += 32) {
            const int b = e / (live * 8), row = (e - b * live * 8) >> 3, c = (e & 7) ^ (row & 7);
            uint16_t* w = reinterpret_cast<uint16_t*>(v + b * kBlock + row * 128 + ((e & 7) << 4));
#pragma unroll 1
            for (int q = 0; q < 8; ++q) {
              const float y = value16<BF16>(w[q]);
              if (fabsf(y) <= 3.4028235e38f) continue;
              atomicMin(&sh.first[i % kItems][y != y ? 0 : y > 0.f ? 1 : 2][b * 64 + c * 8 + q], k * kK + row);
              w[q] = 0;
            }
          }
        }
        tc::fence_proxy_async();
        __syncwarp();
        if (lane == 0) tc::bar_arrive(&sh.v_ready[st]);
      }
      // (the stage is not filled again before it was waited for here)
      if (lane == 0) tc::bar_arrive(&sh.v_free[st]);
    }
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
  }
}

template <int DP, bool BF16>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_kernel(PromptParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                  const __grid_constant__ CUtensorMap map_v) {
  using S = Shape<DP>;
  using Sh = Shared<S::kStages>;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* q_smem = smem;
  unsigned char* k_smem = q_smem + 2 * S::kTile;
  unsigned char* v_smem = k_smem + S::kStages * S::kTile;
  unsigned char* stage = v_smem + S::kStages * S::kTile;
  Sh& sh = *reinterpret_cast<Sh*>(stage + 4 * 32 * 128);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    sh.stop = 0;
    for (int k = 0; k < 2; ++k) {
      tc::bar_init(&sh.q_full[k], 1);
      tc::bar_init(&sh.q_free[k], 1);
      tc::bar_init(&sh.o_full[k], 1);
      tc::bar_init(&sh.o_free[k], 128);
      tc::bar_init(&sh.inv_full[k], 128);
      tc::bar_init(&sh.inv_free[k], 128);
      for (int h = 0; h < 2; ++h) {
        tc::bar_init(&sh.s_full[k][h], 1);
        tc::bar_init(&sh.p_full[k][h], 128);
        tc::bar_init(&sh.o_done[k][h], 1);
      }
    }
    for (int k = 0; k < S::kStages; ++k) {
      tc::bar_init(&sh.k_full[k], 1);
      tc::bar_init(&sh.k_free[k], 2);
      tc::bar_init(&sh.v_full[k], 1);
      tc::bar_init(&sh.v_ready[k], 1);
      tc::bar_init(&sh.v_free[k], 3);
    }
    for (int k = 0; k < kItems; ++k) {
      tc::bar_init(&sh.item_full[k], 1);
      tc::bar_init(&sh.item_free[k], 16);  // every warp
      sh.odd[k] = 0;
    }
    tc::bar_init(&sh.drain, 2);
    tc::bar_fence_init();
  }
  for (int e = threadIdx.x; e < kItems * 3 * 128; e += kThreads) (&sh.first[0][0][0])[e] = kNever;
  pdl_wait();
  if (warp == 12) tc::tmem_alloc(&sh.tmem, 512);
  prompt_list(p, sh.list, Count{p}, p.most);
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  const uint32_t tmem = sh.tmem;
  // registers: 512 threads start with 128 each, four warpgroups split them
  if (warp < 8) {
    tc::setmaxnreg_inc<kRegSoftmax>();
    softmax_role<DP, BF16>(p, sh, tmem, warp >> 2);
  } else if (warp < 12) {
    tc::setmaxnreg_dec<kRegWrite>();
    write_role<DP, BF16>(p, sh, stage, tmem);
  } else {
    tc::setmaxnreg_dec<kRegIssue>();
    if (warp == 13)
      load_role<DP>(p, sh, map_q, map_k, map_v, q_smem, k_smem, v_smem);
    else if (warp == 15)
      look_role<DP, BF16>(p, sh, v_smem);
    else if (tc::elect_one())
      issue_role<DP, BF16>(p, sh, tc::su32(q_smem), tc::su32(k_smem), tc::su32(v_smem), tmem, warp == 14);
  }
  __syncthreads();
  // after a wait that ran out, products and copies may still be in flight (the lane that issued the
  // products is the one whose commit covers them)
  if (sh.stop && (warp == 12 || warp == 14) && tc::elect_one()) {
    tc::mma_commit(&sh.drain);
    tc::bar_wait(&sh.drain, 0, nullptr, kPromptWaitNs);
    for (int k = 0; k < 2 * (2 * S::kStages + 2); ++k) {
      uint64_t* bar = k / 2 < S::kStages ? &sh.k_full[k / 2] : k / 2 < 2 * S::kStages ? &sh.v_full[k / 2 - S::kStages] : &sh.q_full[k / 2 - 2 * S::kStages];
      tc::bar_wait(bar, k & 1, nullptr, kPromptWaitNs / 16);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) prompt_leave(p, gridDim.x, sh.stop);
  if (warp == 12) tc::tmem_dealloc(tmem, 512);
}

// Once per device: the shared memory, and that the register split adds up --
// setmaxnreg.inc waits for registers that only the launch's own can give.
template <int DP, bool BF16>
int launch(const PromptParams& p, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, int grid, cudaStream_t st) {
  using S = Shape<DP>;
  constexpr int smem = (2 + 2 * S::kStages) * S::kTile + 4 * 32 * 128 + (int)sizeof(Shared<S::kStages>);
  static_assert(smem <= 227 * 1024 - 64, "an SM's shared memory");
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return OCCAM_ERR_CUDA;
  if (!((ready.load(std::memory_order_acquire) >> dev) & 1)) {
    cudaFuncAttributes at;
    if (cudaFuncGetAttributes(&at, prompt_kernel<DP, BF16>) != cudaSuccess) return OCCAM_ERR_CUDA;
    if (at.numRegs * kThreads < 256 * kRegSoftmax + 128 * (kRegWrite + kRegIssue)) return OCCAM_ERR_UNSUPPORTED;
    if (cudaFuncSetAttribute(prompt_kernel<DP, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
      return OCCAM_ERR_CUDA;
    ready.fetch_or(uint64_t(1) << dev, std::memory_order_release);
  }
  return launch_after(prompt_kernel<DP, BF16>, dim3((unsigned)grid), kThreads, smem, st, p, mq, mk, mv) && cudaGetLastError() == cudaSuccess
             ? OCCAM_OK
             : OCCAM_ERR_CUDA;
}

template <int DP>
int launch_dtype(const PromptParams& p, bool bf16, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, int grid,
                 cudaStream_t st) {
  return bf16 ? launch<DP, true>(p, mq, mk, mv, grid, st) : launch<DP, false>(p, mq, mk, mv, grid, st);
}

}  // namespace

bool occam::encode_rows(CUtensorMap* m, const void* at, bool bf16, int dim, int heads, int64_t rows, int64_t row, int box_heads,
                        int box_rows, int box_dims) {
  static const PFN_cuTensorMapEncodeTiled_v12000 enc = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool found = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) ==
                           cudaSuccess && q == cudaDriverEntryPointSuccess;
    return found ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f) : nullptr;
  }();
  if (!enc) return false;
  cuuint64_t gdim[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)rows};
  cuuint64_t gstride[2] = {(cuuint64_t)dim * 2, (cuuint64_t)row * 2};
  cuuint32_t box[3] = {(cuuint32_t)box_dims, (cuuint32_t)box_heads, (cuuint32_t)box_rows};
  cuuint32_t es[3] = {1, 1, 1};
  return enc(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(at), gdim, gstride,
             box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, box_dims == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_32B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int occam::prompt_params(const occam_prompt_args* a, void* workspace, size_t workspace_bytes, PromptParams* p) {
  if (!a) return OCCAM_ERR_INVALID_ARG;
  if (a->dtype != OCCAM_BF16 && a->dtype != OCCAM_F16) return OCCAM_ERR_UNSUPPORTED;
  if (a->dim < 8 || a->dim > 128 || a->dim % 8 != 0) return OCCAM_ERR_UNSUPPORTED;
  if (a->total_rows < 0 || a->total_rows > kPromptRows || a->total_keys < 0 || a->total_keys > kPromptRows || a->n < 0 ||
      a->n > (1 << 20) || a->kv_heads < 1 || a->heads < 1 || a->heads > 1024 || a->heads % a->kv_heads != 0 || !(a->scale >= 0.f) ||
      !(a->scale < INFINITY))
    return OCCAM_ERR_INVALID_ARG;
  size_t need = 0;
  const int rc = occam_prompt_workspace_size(a->total_rows, a->total_keys, a->heads, a->kv_heads, &need);
  if (rc != OCCAM_OK) return rc;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < need) return OCCAM_ERR_WORKSPACE;
  if (a->n == 0 || (a->total_rows == 0 && a->total_keys == 0)) return OCCAM_OK;
  if (!a->row_off || !a->key_off) return OCCAM_ERR_INVALID_ARG;
  auto fits = [&](const void* x, int64_t rows, int64_t row, int heads) {
    return rows == 0 || (x && aligned16(x) && (row & 7) == 0 && row >= (int64_t)heads * a->dim && row < (int64_t(1) << 38));
  };
  if (!fits(a->q, a->total_rows, a->q_row, a->heads) || !fits(a->k, a->total_keys, a->k_row, a->kv_heads) ||
      !fits(a->v, a->total_keys, a->v_row, a->kv_heads))
    return OCCAM_ERR_INVALID_ARG;
  p->n = a->n;
  p->H = a->heads;
  p->Hkv = a->kv_heads;
  p->G = a->heads / a->kv_heads;
  p->log2P = 0;
  while (p->log2P < 7 && p->G % (2 << p->log2P) == 0) ++p->log2P;
  p->causal = a->causal ? 1 : 0;
  p->dim = a->dim;
  p->total_rows = a->total_rows;
  p->total_keys = a->total_keys;
  p->row_off = a->row_off;
  p->key_off = a->key_off;
  const double scale = a->scale > 0.f ? (double)a->scale : 1.0 / std::sqrt((double)a->dim);
  p->scale = (float)scale;
  p->scale_log2 = std::max((float)(scale * 1.4426950408889634), kLeastFactor);
  p->status = ws_at<int32_t>(workspace, 0);
  p->counters = ws_at<int32_t>(workspace, 8);
  return OCCAM_OK;
}

bool occam::prompt_meets_inputs(const occam_prompt_args* a, const Extent& x) {
  auto rows = [&](const void* at, int64_t n, int64_t row, int heads) {
    return n > 0 && meet(x, extent(at, n, row, 1, 0, (int64_t)heads * a->dim, 2));
  };
  return rows(a->q, a->total_rows, a->q_row, a->heads) || rows(a->k, a->total_keys, a->k_row, a->kv_heads) ||
         rows(a->v, a->total_keys, a->v_row, a->kv_heads);
}

#define OCCAM_TRY(x)                 \
  do {                               \
    int _rc = (x);                   \
    if (_rc != OCCAM_OK) return _rc; \
  } while (0)

extern "C" int occam_prompt_workspace_size(int64_t total_rows, int64_t total_keys, int32_t heads, int32_t kv_heads, size_t* bytes) {
  if (!bytes || total_rows < 0 || total_rows > kPromptRows || total_keys < 0 || total_keys > kPromptRows || heads < 1 ||
      heads > 1024 || kv_heads < 1 || kv_heads > heads)
    return OCCAM_ERR_INVALID_ARG;
  *bytes = prompt_ws(total_rows, total_keys, heads, kv_heads).total;
  return OCCAM_OK;
}

extern "C" int occam_prompt_attend(const occam_prompt_args* a, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                   occam_stream_t stream) {
  const NvtxRange nvtx("occam_prompt_attend");
  launch_counter() = 0;
  PromptParams p{};
  OCCAM_TRY(prompt_params(a, workspace, workspace_bytes, &p));
  if (a->n == 0 || a->total_rows == 0) return OCCAM_OK;
  const int64_t width = (int64_t)a->heads * a->dim;
  const Extent o = extent(out, a->total_rows, width, 1, 0, width, 2), l = extent(lse, 1, 0, 1, 0, a->total_rows * a->heads * 2, 2);
  if (!out || !aligned16(out) || prompt_meets_inputs(a, o) || (lse && (prompt_meets_inputs(a, l) || meet(o, l)))) return OCCAM_ERR_INVALID_ARG;
  p.out = static_cast<uint16_t*>(out);
  p.lse = lse;
  const bool bf16 = a->dtype == OCCAM_BF16;
  const int per = 256 >> p.log2P, heads = p.H >> p.log2P;
  const int64_t most = (a->total_rows / per + a->n) * heads;
  if (most > (1 << 30)) return OCCAM_ERR_UNSUPPORTED;
  p.most = (int)most;
  CUtensorMap mq, mk, mv;
  // (without any keys the copies have to come from somewhere; what they bring is hidden)
  const bool none = a->total_keys == 0;
  if (!encode_rows(&mq, a->q, bf16, p.dim, p.H, a->total_rows, a->q_row, 1 << p.log2P, 128 >> p.log2P) ||
      !encode_rows(&mk, none ? a->q : a->k, bf16, p.dim, p.Hkv, none ? 1 : a->total_keys, none ? a->q_row : a->k_row, 1, kK) ||
      !encode_rows(&mv, none ? a->q : a->v, bf16, p.dim, p.Hkv, none ? 1 : a->total_keys, none ? a->q_row : a->v_row, 1, kK))
    return OCCAM_ERR_CUDA;
  const int grid = (int)std::min<int64_t>(cache_sms(), most);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (p.dim <= 64) return launch_dtype<64>(p, bf16, mq, mk, mv, grid, st);
  if (p.dim <= 80) return launch_dtype<80>(p, bf16, mq, mk, mv, grid, st);
  return launch_dtype<128>(p, bf16, mq, mk, mv, grid, st);
}
