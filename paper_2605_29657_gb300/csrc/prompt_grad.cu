// prompt_grad.cu -- gradient of a whole prompt's attention: occam_prompt_attend_grad.
//
// With s = scale q.k, p = exp(s - lse), dP = dO V^T and delta = dO.O a row:
//   dV = P^T dO,  dS = P (dP - delta),  dQ = scale dS K,  dK = scale dS^T Q.
// Neither P nor dS goes to memory: two kernels on the fifth-generation tensor cores form them again, one that
// owns keys (dK, dV; 8 D operations a (row, head, key)) and one that owns rows (dQ; 6 D). Every
// sum has one order, the heads of a group included, so results repeat bit for bit; a kernel that
// owned keys alone would do with 10 D in all but add dQ across CTAs. Where there are few tiles of keys their rows are
// divided into up to 8 parts of 12 steps or more, whose sums in fp32 a last launch adds up in order (1,000 rows, 8 heads on one
// key head: 119 -> 61 us; 3,500 rows, 5 on one: 264 -> 134; 2,400 rows, 28 on 4: 265 -> 180).
// Before them a pass over dO and O forms delta; with f16, where dS has no range to spare, also the norms
// that bound it: |dP - delta| <= |dO||V| + |delta|, and dS is held times a power of two a sequence and key head that
// brings that bound under f16's end.
// Bound by the products at 128 dims, by the elementwise chain at 64: 2,048 rows of 8,192 keys, 19 heads: keys 222 us and rows 169 us
// at 128 dims (1,470 and 1,450 TFLOP/s), 107 us rows at 64. With few key heads the longest causal column of key tiles
// is a CTA's whole time: 4,177 rows of 32 heads on 8 key heads 270 us, 236 if it could be divided.
#include <algorithm>
#include <atomic>

#include "nvtx.cuh"
#include "prompt.cuh"

using namespace occam;

namespace {

constexpr int kThreads = 512;
constexpr int kItems = 3;           // items known ahead
constexpr int kRegElement = 160, kRegWrite = 88, kRegIssue = 104;  // 2 x 160 + 88 + 104 = 4 x 128
constexpr int kRowBytes = 128;      // of 64 dims in a block

struct GradParams : PromptParams {
  int most_keys;  // items of tiles of keys, as `most`
  int parts;      // of an item of keys, at most
  float* split;   // [parts, 2, total_keys, kv_heads, dim] sums of dV and dK of divided items
  const uint16_t* o;
  const uint16_t* dout;
  int64_t dout_row, v_row;
  const uint16_t* v;
  uint16_t *dq, *dk, *dv;
  int64_t dq_row, dk_row, dv_row;
  float2* stat;   // [total_rows, heads] lse in log2 units, -delta
  uint4* terms;   // [total_rows, heads, 2] 16-bit terms: four of -lse / scale, four of -delta, eight zeros
  float* norm;    // (f16) [total_rows, heads] |dO|
  float* vnorm;   // (f16) [total_keys, kv_heads] |V|
  float* power;   // (f16) [total_rows, kv_heads], at a sequence's first row: what its dS is held times of
};

template <bool BF16>
__device__ __forceinline__ float2 pair16(uint32_t w) {
  return BF16 ? make_float2(bf16_lo(w), bf16_hi(w)) : __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// A number as a sum of up to four 16-bit terms, each in a unit of its own (see the kernel of keys). f16: a value below 2^31
// is held to 2^-39 or a relative 2^-46; bf16 (24 bits, fp32's range) needs no units.
template <bool BF16>
__device__ __forceinline__ uint2 units4() {
  return BF16 ? make_uint2(pack16<true>(1.f, 1.f), pack16<true>(1.f, 0.f))
              : make_uint2(pack16<false>(32768.f, 32.f), pack16<false>(1.f / 32.f, 1.f / 16384.f));
}
template <bool BF16>
__device__ __forceinline__ uint2 terms4(float x) {
  if (!(fabsf(x) < (BF16 ? 3.3e38f : 2147483648.f)))  // infinities and NaN as they are
    return make_uint2(pack16<BF16>(x != x ? x : x > 0.f ? INFINITY : -INFINITY, 0.f), 0);
  if (BF16) {
    const float a = __bfloat162float(__float2bfloat16_rn(x)), b = __bfloat162float(__float2bfloat16_rn(x - a));
    return make_uint2(pack16<true>(a, b), pack16<true>(x - a - b, 0.f));
  }
  const float a = __half2float(__float2half_rn(x * (1.f / 32768.f))), r0 = fmaf(a, -32768.f, x);
  const float b = __half2float(__float2half_rn(r0 * (1.f / 32.f))), r1 = fmaf(b, -32.f, r0);
  const float c = __half2float(__float2half_rn(r1 * 32.f)), r2 = fmaf(c, -1.f / 32.f, r1);
  return make_uint2(pack16<false>(a, b), pack16<false>(c, r2 * 16384.f));
}

// ---------------------------------------------------------------- delta
// Bound by HBM: dO and O read once. 2^LOG lanes a vector, kVectors vectors' loads of a thread in flight.
constexpr int kVectors = 4;
template <bool BF16, int LOG>
__global__ void __launch_bounds__(256) stat_kernel(GradParams p) {
  pdl_wait();
  constexpr int LANES = 1 << LOG, PER = 256 / LANES;
  const int sub = threadIdx.x & (LANES - 1), first = threadIdx.x >> LOG;
  const bool of_v = blockIdx.y != 0;  // (f16) norms of V
  const int heads = of_v ? p.Hkv : p.H;
  const int64_t vectors = (of_v ? p.total_keys : p.total_rows) * heads;
  const int64_t base = (int64_t)blockIdx.x * (PER * kVectors);
  if (base >= vectors) return;
  const int64_t row0 = base >> 32 ? base / heads : (uint32_t)base / (uint32_t)heads;
  const int head0 = (int)(base - row0 * heads);
  const float inv = 1.f / heads;
  // The vector that this lane writes (sub < 4): the reduction below leaves it there.
  const int mine = ((sub & 1) << 1) | ((sub >> 1) & 1);
  const int64_t to = base + mine * PER + first;
  const bool writes = sub < kVectors && to < vectors;
  const float l = writes && !of_v ? p.lse[to] : 0.f;
  uint4 a[kVectors], b[kVectors];
#pragma unroll
  for (int k = 0; k < kVectors; ++k) {
    // (at < heads + 128 <= 1152: the product is off by 2^-22 of at / heads, a 1 / (2 heads) from the next integer)
    const int at = head0 + k * PER + first, row = (int)((at + 0.5f) * inv);
    a[k] = b[k] = make_uint4(0, 0, 0, 0);
    if (base + k * PER + first < vectors && sub * 8 < p.dim) {
      if (of_v) {
        b[k] = ldg_stream(p.v + (row0 + row) * p.v_row + (at - row * heads) * p.dim + sub * 8);
      } else {
        a[k] = ldg_stream(p.o + (base + k * PER + first) * p.dim + sub * 8);
        b[k] = ldg_stream(p.dout + (row0 + row) * p.dout_row + (at - row * heads) * p.dim + sub * 8);
      }
    }
  }
  float dot[kVectors], sq[kVectors];
#pragma unroll
  for (int k = 0; k < kVectors; ++k) {
    const uint32_t x[4] = {a[k].x, a[k].y, a[k].z, a[k].w}, y[4] = {b[k].x, b[k].y, b[k].z, b[k].w};
    dot[k] = sq[k] = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 u = pair16<BF16>(x[e]), v = pair16<BF16>(y[e]);
      dot[k] = fmaf(u.x, v.x, fmaf(u.y, v.y, dot[k]));
      if (!BF16) sq[k] = fmaf(v.x, v.x, fmaf(v.y, v.y, sq[k]));
    }
  }
  // Exchanges that halve the vectors a lane has and double the lanes it has seen, then the rest of the lanes.
  auto sum = [&](float (&x)[kVectors]) {
#pragma unroll
    for (int n = kVectors / 2, o = 1; n > 0; n >>= 1, o <<= 1) {
#pragma unroll
      for (int k = 0; k < n; ++k) {
        const bool high = sub & o;
        const float give = high ? x[k] : x[k + n], keep = high ? x[k + n] : x[k];
        x[k] = keep + __shfl_xor_sync(0xffffffffu, give, o);
      }
    }
#pragma unroll
    for (int o = kVectors; o < LANES; o <<= 1) x[0] += __shfl_xor_sync(0xffffffffu, x[0], o);
  };
  static_assert(kVectors == 4 && LANES >= 4, "mine");
  sum(dot);
  if (!BF16) sum(sq);
  if (!writes) return;
  if (of_v) {
    p.vnorm[to] = sqrtf(sq[0]);
  } else {
    const float l2 = l == -INFINITY ? INFINITY : l * 1.44269504089f;  // (a row that sees nothing: every p is 0)
    p.stat[to] = make_float2(l2, -dot[0]);
    // (finite in that row: a mask hides its keys there, and an infinity would meet the other product's units of 0)
    const uint2 x = terms4<BF16>(l2 == INFINITY ? 0.f : -l2 / p.scale_log2), y = terms4<BF16>(-dot[0]);
    p.terms[2 * to] = make_uint4(x.x, x.y, y.x, y.y);
    p.terms[2 * to + 1] = make_uint4(0, 0, 0, 0);
    if (!BF16) p.norm[to] = sqrtf(sq[0]);
  }
}

// (f16) One CTA a sequence and key head: the power of two that brings the bound of dS under 2^15.
__global__ void __launch_bounds__(512) power_kernel(GradParams p) {
  __shared__ float sh[3][16];
  pdl_wait();
  const PromptSeq s = prompt_seq(p, blockIdx.x);
  const int h = blockIdx.y;
  if (s.rows == 0) return;
  float m[3] = {0.f, 0.f, 0.f};
  for (int64_t e = threadIdx.x; e < (int64_t)s.rows * p.G; e += 512) {
    const int64_t row = e / p.G, at = (s.row0 + row) * p.H + h * p.G + (e - row * p.G);
    m[0] = fmaxf(m[0], finite_abs(p.norm[at]));
    m[1] = fmaxf(m[1], finite_abs(p.stat[at].y));
  }
  for (int64_t e = threadIdx.x; e < s.keys; e += 512) m[2] = fmaxf(m[2], finite_abs(p.vnorm[(s.key0 + e) * p.Hkv + h]));
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    m[k] = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m[k])));
    if ((threadIdx.x & 31) == 0) sh[k][threadIdx.x >> 5] = m[k];
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 0; k < 3; ++k)
      for (int w = 0; w < 16; ++w) m[k] = fmaxf(m[k], sh[k][w]);
    const float bound = fminf(fmaf(m[0], m[2], m[1]), 3e38f);
    int e = 0;
    if (bound > 0.f) e = 14 - ((__float_as_int(bound) >> 23) - 127);  // bound 2^e < 2^15
    p.power[s.row0 * p.Hkv + h] = __int_as_float((min(max(e, -100), 100) + 127) << 23);
  }
}

#define WAIT(bar, parity) PROMPT_WAIT(bar, parity)

// f16: P is held 2^14 times as large (it is at most 1, up to the rounding of lse), so that what is 2^-28 of the
// largest still has 11 bits.
template <bool BF16>
struct Lift {
  static constexpr float kLog2 = BF16 ? 0.f : 14.f, kBack = BF16 ? 1.f : 1.f / 16384.f;
};

// The 16-bit results of 32 rows, of a lane each, over shared memory to rows of global memory: 16 values at a time are
// put by put16, whole 64-dim blocks written by flush. to(row) gives a row's address, null if it is not there.
struct RowWriter {
  unsigned char* stage;  // 32 x 128 bytes of this warp
  int lane;
  __device__ __forceinline__ void put16(int c, const uint32_t (&w)[8]) const {
#pragma unroll
    for (int e = 0; e < 2; ++e)
      *reinterpret_cast<uint4*>(stage + lane * 128 + (((c / 8 + e) ^ (lane & 7)) << 4)) =
          make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
  }
  template <class To>
  __device__ __forceinline__ void flush(int block, int pieces, const To& to) const {
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int rr = e * 4 + lane / 8, c = lane % 8;
      const uint4 v = *reinterpret_cast<const uint4*>(stage + rr * 128 + ((c ^ (rr & 7)) << 4));
      uint16_t* at = to(rr);
      if (at && block * 8 + c < pieces) *reinterpret_cast<uint4*>(at + block * 64 + c * 8) = v;
    }
    __syncwarp();
  }
};
template <bool BF16>
__device__ __forceinline__ void scale_pack(const uint32_t (&o)[16], float f, uint32_t (&w)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = pack16<BF16>(__uint_as_float(o[2 * e]) * f, __uint_as_float(o[2 * e + 1]) * f);
}

// ================================================================ dK and dV
// An item is a tile of 128 keys of one key head; its steps are blocks of 64 query rows (64 / P tokens x P heads),
// first rows that see it on, for every head of the group. Scores are taken transposed, S^T = K Q^T and dP^T = V dO^T, a
// key a lane, so that P^T and dS^T are the first operands of dV += P^T dO and dK += dS^T Q from tensor memory.
// Even and odd steps have tensor memory, an issuing warp and a warpgroup of their own: while one's scores are
// turned into P and dS, the other's products run. The sums are added to in the order of the steps (a step's product
// waits for the one before it; the scores issued in between keep the tensor cores busy).
// A row's lse and delta are constants of a column here. They come in as 16 more dims of both products: every row
// brings -lse / scale and -delta as sums of up to four 16-bit terms, the first operand has those terms' units (of
// the one in S^T, of the other in dP^T), so that S^T and dP^T arrive as what the exponential and the product want.
namespace keys {

constexpr int kQ = 64;                  // query rows of a step
constexpr int kMoreBytes = kQ * 32;     // of the rows' 16 more dims
constexpr int kUnitBytes = 128 * 32;    // of the first operand's

template <int DP>
struct Shape {
  static constexpr int kBlocks = DP > 64 ? 2 : 1;
  static constexpr int kTile = kBlocks * 128 * kRowBytes;  // bytes of 128 rows
  static constexpr int kHalf = kTile / 2;                  // and of 64
  static constexpr int kStages = DP > 64 ? 4 : 6;
};

template <int STAGES>
struct Shared {
  uint64_t kv_full, kv_free, full[STAGES], ready[STAGES], free[STAGES], s_full[2], dp_full[2], p_full[2], ds_full[2], added[2], o_full,
      o_free, item_full[kItems], item_free[kItems], drain;
  PromptItem item[kItems];  // tile: of keys; hb: key head; nk[0]: the first block of rows; nk[1]: 0, or 1 at the end
  uint32_t tmem;
  int stop;
  PromptList list;
};

struct Count {
  const GradParams& p;
  __device__ __forceinline__ int operator()(const PromptSeq& s) const { return (s.keys / 128 + (s.keys % 128 != 0)) * p.Hkv * p.parts; }
};
// A tile's first block of rows, blocks of a head block, and steps; parts of so many steps at least (1,000 rows of 8 heads
// on one key head: 58 us, 64 with 16, 83 with 32; 300 rows of 32 on 8: 39, 43 with 8; finding the tiles to add up by their
// items takes 1 us more since).
constexpr int kPartSteps = 12;
struct Tile {
  int first, blocks, steps, parts;

  __device__ __forceinline__ Tile(const GradParams& p, const PromptSeq& s, int tile, int log_p) {
    const int log_t = 6 - log_p;
    first = (p.causal ? max(tile * 128 - (s.keys - s.rows), 0) : 0) >> log_t;
    blocks = max(((s.rows + (1 << log_t) - 1) >> log_t) - first, 0);
    steps = blocks * (p.G >> log_p);
    parts = min(max(steps / kPartSteps, 1), p.parts);
  }
};

// A walk over an item's steps: blocks of tokens, head block by head block.
struct Steps {
  int head, tok;  // first head, first token
  int tok0, tokens, more;

  __device__ __forceinline__ Steps(const GradParams& p, const PromptItem& it, int log_p) {
    tokens = 1 << (6 - log_p);
    more = it.rows;
    tok0 = it.nk[0] << (6 - log_p);
    const int blocks = max(((it.rows + tokens - 1) >> (6 - log_p)) - it.nk[0], 1), skip = it.step0 / blocks;
    tok = tok0 + (it.step0 - skip * blocks) * tokens;
    head = it.hb * p.G + (skip << log_p);
  }
  __device__ __forceinline__ void next(int log_p) {
    tok += tokens;
    if (tok >= more) {
      tok = tok0;
      head += 1 << log_p;
    }
  }
};

template <int DP, class Sh>
__device__ __forceinline__ void load_role(const GradParams& p, Sh& sh, int log_p, const CUtensorMap& map_q, const CUtensorMap& map_do,
                                          const CUtensorMap& map_k, const CUtensorMap& map_v, const CUtensorMap& map_terms,
                                          unsigned char* k_smem, unsigned char* v_smem, unsigned char* q_smem, unsigned char* more) {
  using S = Shape<DP>;
  const int lane = threadIdx.x & 31;
  uint32_t n = 0, turn = 1;
  int st = 0;
  for (uint32_t i = 0;; ++i) {
    WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
    const PromptItem it = sh.item[i % kItems];
    if (it.nk[1]) return;
    if (it.steps > 0) {
      const int key = (int)(it.key0 + (int64_t)it.tile * 128);
      WAIT(sh.kv_free, (n & 1) ^ 1);
      ++n;
      if (lane == 0) {
        tc::bar_expect_tx(&sh.kv_full, 2 * S::kTile);
        for (int b = 0; b < S::kBlocks; ++b) {
          tc::tma_load_3d(k_smem + b * 128 * kRowBytes, &map_k, b * 64, it.hb, key, &sh.kv_full);
          tc::tma_load_3d(v_smem + b * 128 * kRowBytes, &map_v, b * 64, it.hb, key, &sh.kv_full);
        }
      }
    }
    Steps at(p, it, log_p);
    const int row = (int)it.row0;
#pragma unroll 1
    for (int k = 0; k < it.steps; ++k, at.next(log_p)) {
      WAIT(sh.free[st], turn);
      if (lane == 0) {
        tc::bar_expect_tx(&sh.full[st], S::kTile + kMoreBytes);  // 64 rows of Q and of dO
        tc::tma_load_3d(more + st * kMoreBytes, &map_terms, 0, at.head, row + at.tok, &sh.full[st]);
        unsigned char* to = q_smem + st * S::kTile;
        for (int b = 0; b < S::kBlocks; ++b) {
          tc::tma_load_3d(to + b * kQ * kRowBytes, &map_q, b * 64, at.head, row + at.tok, &sh.full[st]);
          tc::tma_load_3d(to + S::kHalf + b * kQ * kRowBytes, &map_do, b * 64, at.head, row + at.tok, &sh.full[st]);
        }
      }
      __syncwarp();
      if (++st == S::kStages) st = 0, turn ^= 1;
    }
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
    __syncwarp();
  }
}

// Rows past the sequence's end become zeros, terms and all: P is finite there, dP is 0.
template <int DP, class Sh>
__device__ __forceinline__ void look_role(const GradParams& p, Sh& sh, int log_p, unsigned char* q_smem, unsigned char* more) {
  using S = Shape<DP>;
  const int lane = threadIdx.x & 31;
  PromptTaker taker;
  uint32_t told = 0;
  auto tell = [&]() -> bool {
    PromptItem& it = sh.item[told % kItems];
    if (!prompt_wait(&sh.item_free[told % kItems], ((told / kItems) & 1) ^ 1, &sh.stop)) return false;
    const int place = taker.take(p, sh.list, Count{p});
    const PromptSeq& s = taker.s;
    if (place >= 0) {
      const int tile = place / (p.Hkv * p.parts), at = place - tile * (p.Hkv * p.parts), hb = at / p.parts, part = at - hb * p.parts;
      const Tile x(p, s, tile, log_p);
      const int a = (int)((int64_t)x.steps * part / x.parts), b = (int)((int64_t)x.steps * (part + 1) / x.parts);
      if (lane == 0) {
        it.row0 = s.row0;
        it.key0 = s.key0;
        it.rows = s.rows;
        it.keys = s.keys;
        it.tile = tile;
        it.hb = hb;
        it.steps = part < x.parts ? b - a : 0;
        it.nk[0] = x.first;
        it.nk[1] = 0;
        it.step0 = part < x.parts ? a : 0;
        it.part = part >= x.parts ? -2 : x.parts > 1 ? part : -1;
      }
    } else if (lane == 0) {
      it.steps = 0;
      it.nk[1] = 1;
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
    if (sh.item[i % kItems].nk[1]) return;
    if (!tell()) return;  // the next one, while the first copies are under way
    const int steps = sh.item[i % kItems].steps, rows = sh.item[i % kItems].rows, first = sh.item[i % kItems].nk[0];
    const int log_t = 6 - log_p, blocks = ((rows + (1 << log_t) - 1) >> log_t) - first;
    const int last = (rows & ((1 << log_t) - 1)) << log_p;  // rows of the last block of tokens, 0: it is whole
    int block = sh.item[i % kItems].step0 % max(blocks, 1);
#pragma unroll 1
    for (int k = 0; k < steps; ++k, ++j) {
      const int st = j % S::kStages;
      WAIT(sh.full[st], (j / S::kStages) & 1);
      if (++block == blocks) {
        block = 0;
        if (last) {
#pragma unroll 1
          for (int b = 0; b < 2 * S::kBlocks; ++b) {
            uint4* piece = reinterpret_cast<uint4*>(q_smem + st * S::kTile + b * kQ * kRowBytes);
            for (int e = last * 8 + lane; e < kQ * 8; e += 32) piece[e] = make_uint4(0, 0, 0, 0);
          }
          uint4* row = reinterpret_cast<uint4*>(more + st * kMoreBytes);
          for (int e = last * 2 + lane; e < kQ * 2; e += 32) row[e] = make_uint4(0, 0, 0, 0);
          tc::fence_proxy_async();
          __syncwarp();
          if (lane == 0) tc::bar_arrive(&sh.ready[st]);
        }
      }
      // (the stage is not filled again before it was waited for here)
      if (lane == 0) tc::bar_arrive(&sh.free[st]);
    }
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
  }
}

// The steps of parity b. After step j's P: dV += P^T dO, then S^T of step j + 2 in its place; after its dS: dK += dS^T Q and
// dP^T of step j + 2.
template <int DP, bool BF16, class Sh>
__device__ __forceinline__ void issue_role(const GradParams& p, Sh& sh, uint32_t k_smem, uint32_t v_smem, uint32_t q_smem, uint32_t units,
                                           uint32_t more, uint32_t tmem, int log_p, uint32_t b) {
  using S = Shape<DP>;
  constexpr uint32_t id_s = tc::idesc16(BF16, 128, kQ, false), id_o = tc::idesc16(BF16, 128, DP, true);
  const uint64_t kmajor = tc::sdesc_sw128(0), mnmajor = tc::sdesc_mn_sw128(0, kQ * kRowBytes), narrow = tc::sdesc_sw32(0);
  const uint32_t km = tc::desc_hi(kmajor), mn = tc::desc_hi(mnmajor), nm = tc::desc_hi(narrow);
  const uint32_t dk = (uint32_t)kmajor + (k_smem >> 4), dv = (uint32_t)kmajor + (v_smem >> 4);
  const uint32_t dq = (uint32_t)kmajor + (q_smem >> 4), dqt = (uint32_t)mnmajor + (q_smem >> 4);
  // (Both 16-byte pieces of a row of units are the same, and one of a row of terms is 0: the order in which the
  // swizzle puts them does not matter.)
  const uint32_t du = (uint32_t)narrow + (units >> 4), dm = (uint32_t)narrow + (more >> 4);
  const uint32_t s_at = tmem + b * 128, dp_at = s_at + 64, dv_at = tmem + 256, dk_at = tmem + 384;
  // a walk over the steps of this parity
  uint32_t i = 0, j = b;       // items begun; the next own step
  uint32_t base = 0, end = 0;  // the present item's steps
  uint32_t n_kv = 0, kv = 0;   // items with steps: begun; whose keys and values were waited for
  uint32_t done = 0;           // own steps so far
  uint32_t looked = 0;         // a bit a stage: how often (mod 2) its rows were looked at
  int block = 0, blocks = 1;   // of the next own step; in a head block
  bool ragged = false;         // a head block's last block has rows past the end
  struct {
    bool any, first, last;
    uint32_t stage, j, items;
  } was = {false, false, false, 0, 0, 0};
  for (;;) {
    // Step j's item: one item further at most before the products of the step before are issued (the loader
    // knows one ahead; more may wait for those very products)
    bool over = false, have = j < end;
    if (!have) {
      // The item's keys and values are done with once the scores issued so far are -- and have come: given back before, by the
      // warp without a step here, the next ones could come before it looked for these, and two phases on a wait does not end.
      for (; kv < n_kv; ++kv) WAIT(sh.kv_full, kv & 1);
      if (end > base) tc::mma_commit(&sh.kv_free);
      if (i > 0) tc::bar_arrive(&sh.item_free[(i - 1) % kItems]);
      WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
      over = sh.item[i % kItems].nk[1] != 0;
      base = end;
      if (!over) {
        const PromptItem& x = sh.item[i % kItems];
        const int log_t = 6 - log_p;
        end = base + x.steps;
        blocks = max(((x.rows + (1 << log_t) - 1) >> log_t) - x.nk[0], 1);
        block = (int)(j - base) + x.step0 % blocks;  // (past the last one: below)
        ragged = (x.rows & ((1 << log_t) - 1)) != 0;
      }
      if (end > base) ++n_kv;
      ++i;
      have = j < end;
    }
    const uint32_t st = j % S::kStages;
    if (was.any) {
      WAIT(sh.p_full[b], (done - 1) & 1);
      if (was.j > 0) WAIT(sh.added[b ^ 1], ((was.j - 1) >> 1) & 1);  // the step before it
      if (was.first) WAIT(sh.o_free, (was.items & 1) ^ 1);           // (after that: the items before have begun)
      tc::fence_after();
      {
        const uint32_t d = dqt + was.stage * (S::kTile >> 4) + (S::kHalf >> 4);
#pragma unroll
        for (int q = 0; q < kQ / 16; ++q)
          tc::mma16_ts(dv_at, s_at + q * 8, d + q * (16 * kRowBytes >> 4), mn, id_o, q > 0 || !was.first);
      }
    }
    if (have) {
      for (; kv < n_kv; ++kv) WAIT(sh.kv_full, kv & 1);
      WAIT(sh.full[st], (j / S::kStages) & 1);
      while (block >= blocks) block -= blocks;
      if (ragged && block == blocks - 1) {
        WAIT(sh.ready[st], (looked >> st) & 1);
        looked ^= 1u << st;
      }
      block += 2;
      tc::fence_after();
      {
        const uint32_t d = dq + st * (S::kTile >> 4);
#pragma unroll
        for (int q = 0; q < DP / 16; ++q)
          tc::mma16_ss(s_at, dk + (q >> 2) * (128 * kRowBytes >> 4) + (q & 3) * 2, km,
                       d + (q >> 2) * (kQ * kRowBytes >> 4) + (q & 3) * 2, km, id_s, q > 0);
        tc::mma16_ss(s_at, du, nm, dm + st * (kMoreBytes >> 4), nm, id_s, true);
        tc::mma_commit(&sh.s_full[b]);
      }
    }
    if (was.any) {
      WAIT(sh.ds_full[b], (done - 1) & 1);
      tc::fence_after();
      {
        const uint32_t d = dqt + was.stage * (S::kTile >> 4);
#pragma unroll
        for (int q = 0; q < kQ / 16; ++q)
          tc::mma16_ts(dk_at, dp_at + q * 8, d + q * (16 * kRowBytes >> 4), mn, id_o, q > 0 || !was.first);
        tc::mma_commit(&sh.added[b]);
        tc::mma_commit(&sh.free[was.stage]);
        if (was.last) tc::mma_commit(&sh.o_full);
      }
    }
    if (over) return;
    if (!have) {
      was.any = false;
      continue;
    }
    {
      const uint32_t d = dq + st * (S::kTile >> 4) + (S::kHalf >> 4);
#pragma unroll
      for (int q = 0; q < DP / 16; ++q)
        tc::mma16_ss(dp_at, dv + (q >> 2) * (128 * kRowBytes >> 4) + (q & 3) * 2, km,
                     d + (q >> 2) * (kQ * kRowBytes >> 4) + (q & 3) * 2, km, id_s, q > 0);
      tc::mma16_ss(dp_at, du + (kUnitBytes >> 4), nm, dm + st * (kMoreBytes >> 4), nm, id_s, true);
      tc::mma_commit(&sh.dp_full[b]);
    }
    was.any = true;
    was.first = j == base;
    was.last = j + 1 == end;
    was.stage = st;
    was.j = j;
    was.items = n_kv - 1;  // items with steps before this one
    ++done;
    j += 2;
  }
}

// A key a thread: P^T and dS^T of the steps of parity b
template <int DP, bool BF16, class Sh>
__device__ __forceinline__ void element_role(const GradParams& p, Sh& sh, int log_p, uint32_t tmem, uint32_t b) {
  const int r = threadIdx.x & 127, lane = threadIdx.x & 31;
  const uint32_t s_at = tmem + b * 128 + ((uint32_t)(r & ~31) << 16), dp_at = s_at + 64;
  const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
  uint32_t j = 0, done = 0;
  for (uint32_t i = 0;; ++i) {
    WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
    const PromptItem it = sh.item[i % kItems];
    if (it.nk[1]) return;
    const int key = it.tile * 128 + r, ahead = it.keys - it.rows;  // keys before the first row's own
    const float power = BF16 || it.steps == 0 ? 1.f : p.power[it.row0 * p.Hkv + it.hb] * Lift<BF16>::kBack;
    Steps at(p, it, log_p);
#pragma unroll 1
    for (int k = 0; k < it.steps; ++k, ++j, at.next(log_p)) {
      if ((j & 1) != b) continue;
      WAIT(sh.s_full[b], done & 1);
      tc::fence_after();
      uint32_t v[64];
      tc::tmem_ld64(s_at, v);
      tc::wait_ld64(v);
      float pr[64];
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const float2 s = make_float2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
        const float2 y = BF16 ? tc::mul2(s, scale2) : tc::fma2(s, scale2, make_float2(Lift<BF16>::kLog2, Lift<BF16>::kLog2));
        pr[2 * e] = fast_exp2(y.x);
        pr[2 * e + 1] = fast_exp2(y.y);
      }
      // keys that some row of the block does not see (all keys past the sequence's end are nobody's: their rows are not written)
      if (PROMPT_RARE(p.causal && it.tile * 128 + 127 > ahead + at.tok)) {
        const int lo = min(max(key - ahead - at.tok, 0), kQ) << log_p;  // the first row of the block that sees this key
#pragma unroll
        for (int e = 0; e < 64; ++e) pr[e] = e < lo ? 0.f : pr[e];
      }
      {
        uint32_t pk[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) pk[e] = pack16<BF16>(pr[2 * e], pr[2 * e + 1]);
        tc::tmem_st32(s_at, pk);
      }
      tc::tmem_wait_st();
      tc::fence_before();
      tc::bar_arrive(&sh.p_full[b]);
      // Rows that see one key (the first one): p is 1 whatever the score, so dS is 0, not what two sums of the same products
      // leave of one another.
      const int one = -(ahead + at.tok);  // the block's token that sees one key of a causal sequence
      if (PROMPT_RARE(p.causal ? it.tile == 0 && one >= 0 && one < at.tokens : it.keys == 1)) {
        const int lo = p.causal ? one << log_p : 0, hi = p.causal ? (one + 1) << log_p : kQ;
#pragma unroll
        for (int e = 0; e < 64; ++e) pr[e] = e >= lo && e < hi ? 0.f : pr[e];
      }
      WAIT(sh.dp_full[b], done & 1);
      tc::fence_after();
      tc::tmem_ld64(dp_at, v);
      tc::wait_ld64(v);
      uint32_t pk[32];
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        float2 y = tc::mul2(make_float2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), make_float2(pr[2 * e], pr[2 * e + 1]));
        if (!BF16) y = tc::mul2(y, make_float2(power, power));
        pk[e] = pack16<BF16>(y.x, y.y);
      }
      tc::tmem_st32(dp_at, pk);
      tc::tmem_wait_st();
      tc::fence_before();
      tc::bar_arrive(&sh.ds_full[b]);
      ++done;
    }
    __syncwarp();
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
  }
}

template <int DP, bool BF16, class Sh>
__device__ __forceinline__ void write_role(const GradParams& p, Sh& sh, unsigned char* stage, uint32_t tmem) {
  const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31;
  const uint32_t lanes = (uint32_t)(warp * 32) << 16;
  const RowWriter writer{stage + warp * (32 * 128), lane};
  uint32_t n = 0;
  for (uint32_t i = 0;; ++i) {
    WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
    const PromptItem it = sh.item[i % kItems];
    if (it.nk[1]) return;
    if (it.steps > 0) {
      WAIT(sh.o_full, n & 1);
      tc::fence_after();
      ++n;
    }
    const float back = BF16 || it.steps == 0 ? 1.f : 1.f / p.power[it.row0 * p.Hkv + it.hb];
    if (it.part >= 0) {
      // a part's sums as they are, a key a lane (added up and rounded by split_kernel)
      const int64_t key = (int64_t)it.tile * 128 + warp * 32 + lane;
      const bool there = key < it.keys && in_bounds(it.key0 + key < p.total_keys && it.part < p.parts, p.status, kSitePromptRow);
#pragma unroll 1
      for (int which = 0; which < 2; ++which) {
        float* to = p.split + ((((int64_t)it.part * 2 + which) * p.total_keys + it.key0 + key) * p.Hkv + it.hb) * p.dim;
        const float f = which ? p.scale * back : Lift<BF16>::kBack;
#pragma unroll 1
        for (int c = 0; c < DP; c += 16) {
          uint32_t o[16];
          tc::tmem_ld16(tmem + 256 + which * 128 + lanes + c, o);
          if (there) {
#pragma unroll
            for (int e = 0; e < 16; e += 4)
              if (c + e < p.dim)
                *reinterpret_cast<float4*>(to + c + e) = make_float4(__uint_as_float(o[e]) * f, __uint_as_float(o[e + 1]) * f,
                                                                     __uint_as_float(o[e + 2]) * f, __uint_as_float(o[e + 3]) * f);
          }
          __syncwarp();
        }
      }
      tc::fence_before();
      tc::bar_arrive(&sh.o_free);
    }
#pragma unroll 1
    for (int which = it.part == -1 ? 0 : 2; which < 2; ++which) {
      uint16_t* base = which ? p.dk : p.dv;
      const int64_t row = which ? p.dk_row : p.dv_row;
      const float f = which ? p.scale * back : Lift<BF16>::kBack;
#pragma unroll 1
      for (int blk = 0; blk < Shape<DP>::kBlocks; ++blk) {
        const int cols = min(DP - blk * 64, 64);
#pragma unroll 1
        for (int c = 0; c < cols; c += 16) {
          uint32_t o[16], w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
          if (it.steps > 0) {
            tc::tmem_ld16(tmem + 256 + which * 128 + lanes + blk * 64 + c, o);
            scale_pack<BF16>(o, f, w);
          }
          writer.put16(c, w);
        }
        if (which && blk == Shape<DP>::kBlocks - 1 && it.steps > 0) {
          tc::fence_before();
          tc::bar_arrive(&sh.o_free);
        }
        writer.flush(blk, p.dim / 8, [&](int rr) -> uint16_t* {
          const int64_t key = (int64_t)it.tile * 128 + warp * 32 + rr;
          return key < it.keys && in_bounds(it.key0 + key < p.total_keys, p.status, kSitePromptRow)
                     ? base + (it.key0 + key) * row + it.hb * p.dim
                     : nullptr;
        });
      }
    }
    __syncwarp();
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
  }
}

template <int DP, bool BF16>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_keys_kernel(GradParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_do,
                       const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                       const __grid_constant__ CUtensorMap map_terms) {
  using S = Shape<DP>;
  using Sh = Shared<S::kStages>;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* k_smem = smem;
  unsigned char* v_smem = k_smem + S::kTile;
  unsigned char* q_smem = v_smem + S::kTile;
  unsigned char* stage = q_smem + S::kStages * S::kTile;
  unsigned char* units = stage + 4 * 32 * 128;
  unsigned char* more = units + 2 * kUnitBytes;
  Sh& sh = *reinterpret_cast<Sh*>(more + S::kStages * kMoreBytes);
  const int warp = threadIdx.x >> 5, log_p = min(p.log2P, 6);
  {
    static_assert(2 * kUnitBytes == kThreads * 16, "a piece a thread");
    const uint2 u = units4<BF16>();
    reinterpret_cast<uint4*>(units)[threadIdx.x] = threadIdx.x < kThreads / 2 ? make_uint4(u.x, u.y, 0, 0) : make_uint4(0, 0, u.x, u.y);
  }
  tc::fence_proxy_async();
  if (threadIdx.x == 0) {
    sh.stop = 0;
    tc::bar_init(&sh.kv_full, 1);
    tc::bar_init(&sh.kv_free, 2);
    for (int k = 0; k < S::kStages; ++k) {
      tc::bar_init(&sh.full[k], 1);
      tc::bar_init(&sh.ready[k], 1);
      tc::bar_init(&sh.free[k], 2);
    }
    for (int k = 0; k < 2; ++k) {
      tc::bar_init(&sh.s_full[k], 1);
      tc::bar_init(&sh.dp_full[k], 1);
      tc::bar_init(&sh.p_full[k], 128);
      tc::bar_init(&sh.ds_full[k], 128);
      tc::bar_init(&sh.added[k], 1);
    }
    tc::bar_init(&sh.o_full, 1);
    tc::bar_init(&sh.o_free, 128);
    for (int k = 0; k < kItems; ++k) {
      tc::bar_init(&sh.item_full[k], 1);
      tc::bar_init(&sh.item_free[k], 16);  // every warp
    }
    tc::bar_init(&sh.drain, 2);
    tc::bar_fence_init();
  }
  pdl_wait();
  if (warp == 12) tc::tmem_alloc(&sh.tmem, 512);
  prompt_list(p, sh.list, Count{p}, p.most_keys);
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  const uint32_t tmem = sh.tmem;
  if (warp < 8) {
    tc::setmaxnreg_inc<kRegElement>();
    element_role<DP, BF16>(p, sh, log_p, tmem, warp >> 2);
  } else if (warp < 12) {
    tc::setmaxnreg_dec<kRegWrite>();
    write_role<DP, BF16>(p, sh, stage, tmem);
  } else {
    tc::setmaxnreg_dec<kRegIssue>();
    if (warp == 13)
      load_role<DP>(p, sh, log_p, map_q, map_do, map_k, map_v, map_terms, k_smem, v_smem, q_smem, more);
    else if (warp == 15)
      look_role<DP>(p, sh, log_p, q_smem, more);
    else if (tc::elect_one())
      issue_role<DP, BF16>(p, sh, tc::su32(k_smem), tc::su32(v_smem), tc::su32(q_smem), tc::su32(units), tc::su32(more), tmem, log_p,
                           warp == 14);
  }
  __syncthreads();
  // after a wait that ran out, products and copies may still be in flight
  if (sh.stop && (warp == 12 || warp == 14) && tc::elect_one()) {
    tc::mma_commit(&sh.drain);
    tc::bar_wait(&sh.drain, 0, nullptr, kPromptWaitNs);
    for (int k = 0; k < 2 * (S::kStages + 1); ++k)
      tc::bar_wait(k / 2 < S::kStages ? &sh.full[k / 2] : &sh.kv_full, k & 1, nullptr, kPromptWaitNs / 16);
  }
  __syncthreads();
  if (threadIdx.x == 0) prompt_leave(p, gridDim.x, sh.stop);
  if (warp == 12) tc::tmem_dealloc(tmem, 512);
}

}  // namespace keys

// ================================================================ dQ
// An item is 256 query rows, two tiles of 128 as in the forward pass; its steps are blocks of 64 keys. S = Q K^T and
// dP = dO V^T a row a lane, dS in the place of dP, dQ += dS K. Each row tile has an issuing warp and a
// warpgroup: the next step's scores are multiplied as soon as a step's have been read, its dP behind dQ; and while one
// tile's dS is formed, the other's products run.
namespace rows {

constexpr int kKeys = 64;

template <int DP>
struct Shape {
  static constexpr int kBlocks = DP > 64 ? 2 : 1;
  static constexpr int kTile = kBlocks * 128 * kRowBytes;  // bytes of 128 rows
  static constexpr int kHalf = kTile / 2;                  // and of 64
  static constexpr int kStagesK = DP > 64 ? 3 : 4;         // (keys are held for two steps)
  static constexpr int kStagesV = DP > 64 ? 2 : 4;
};

template <int KS, int VS>
struct Shared {
  uint64_t q_full[2], q_free[2], k_full[KS], k_ready[KS], k_free[KS], v_full[VS], v_free[VS], s_full[2], s_read[2], dp_full[2],
      ds_full[2], o_full[2], o_free[2], item_full[kItems], item_free[kItems], drain;
  PromptItem item[kItems];
  uint32_t tmem;
  int stop;
  PromptList list;
};

struct Count {
  const GradParams& p;
  __device__ __forceinline__ int operator()(const PromptSeq& s) const {
    const int per = 256 >> p.log2P;
    return (s.rows / per + (s.rows % per != 0)) * (p.H >> p.log2P);
  }
};
__device__ __forceinline__ int key_steps(const GradParams& p, const PromptSeq& s, int tok_last) {
  const int lim = min(prompt_limit(p, s.rows, s.keys, tok_last), s.keys);
  return max((lim + kKeys - 1) / kKeys, 1);
}

template <int DP, class Sh>
__device__ __forceinline__ void load_role(const GradParams& p, Sh& sh, const CUtensorMap& map_q, const CUtensorMap& map_do,
                                          const CUtensorMap& map_k, const CUtensorMap& map_v, unsigned char* q_smem,
                                          unsigned char* do_smem, unsigned char* k_smem, unsigned char* v_smem) {
  using S = Shape<DP>;
  const int lane = threadIdx.x & 31;
  uint32_t j = 0, nq[2] = {0, 0};
  for (uint32_t i = 0;; ++i) {
    WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
    const PromptItem it = sh.item[i % kItems];
    if (it.steps == 0) return;
    const int tt = 128 >> p.log2P, head = it.hb << p.log2P, kv = head / p.G;
    for (int k = 0; k < it.steps; ++k, ++j) {
      const int st = j % S::kStagesK, sv = j % S::kStagesV;
      const int key = (int)(it.key0 + (int64_t)k * kKeys);
      WAIT(sh.k_free[st], ((j / S::kStagesK) & 1) ^ 1);
      if (lane == 0) {
        tc::bar_expect_tx(&sh.k_full[st], S::kHalf);
        for (int b = 0; b < S::kBlocks; ++b)
          tc::tma_load_3d(k_smem + st * S::kHalf + b * kKeys * kRowBytes, &map_k, b * 64, kv, key, &sh.k_full[st]);
      }
      if (k == 0) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (it.nk[t] == 0) continue;
          WAIT(sh.q_free[t], (nq[t] & 1) ^ 1);
          ++nq[t];
          if (lane == 0) {
            const int row = (int)(it.row0 + (int64_t)(it.tile * 2 + t) * tt);
            tc::bar_expect_tx(&sh.q_full[t], 2 * S::kTile);
            for (int b = 0; b < S::kBlocks; ++b) {
              tc::tma_load_3d(q_smem + t * S::kTile + b * 128 * kRowBytes, &map_q, b * 64, head, row, &sh.q_full[t]);
              tc::tma_load_3d(do_smem + t * S::kTile + b * 128 * kRowBytes, &map_do, b * 64, head, row, &sh.q_full[t]);
            }
          }
        }
      }
      WAIT(sh.v_free[sv], ((j / S::kStagesV) & 1) ^ 1);
      if (lane == 0) {
        tc::bar_expect_tx(&sh.v_full[sv], S::kHalf);
        for (int b = 0; b < S::kBlocks; ++b)
          tc::tma_load_3d(v_smem + sv * S::kHalf + b * kKeys * kRowBytes, &map_v, b * 64, kv, key, &sh.v_full[sv]);
      }
      __syncwarp();
    }
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
    __syncwarp();
  }
}

// Keys past the sequence's end become zeros: dS is 0 there, but what lies behind may be anything.
template <int DP, class Sh>
__device__ __forceinline__ void look_role(const GradParams& p, Sh& sh, unsigned char* k_smem) {
  using S = Shape<DP>;
  const int lane = threadIdx.x & 31;
  PromptTaker taker;
  uint32_t told = 0;
  auto tell = [&]() -> bool {
    PromptItem& it = sh.item[told % kItems];
    if (!prompt_wait(&sh.item_free[told % kItems], ((told / kItems) & 1) ^ 1, &sh.stop)) return false;
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
    const int steps = sh.item[i % kItems].steps, keys = sh.item[i % kItems].keys;
    if (steps == 0) return;
    if (!tell()) return;  // the next one, while the first copies are under way
    const int whole = keys / kKeys;
#pragma unroll 1
    for (int k = 0; k < steps; ++k, ++j) {
      const int st = j % S::kStagesK, live = max(keys - k * kKeys, 0);
      WAIT(sh.k_full[st], (j / S::kStagesK) & 1);
      if (k >= whole) {
#pragma unroll 1
        for (int b = 0; b < S::kBlocks; ++b) {
          uint4* piece = reinterpret_cast<uint4*>(k_smem + st * S::kHalf + b * kKeys * kRowBytes);
          for (int e = live * 8 + lane; e < kKeys * 8; e += 32) piece[e] = make_uint4(0, 0, 0, 0);
        }
        tc::fence_proxy_async();
        __syncwarp();
        if (lane == 0) tc::bar_arrive(&sh.k_ready[st]);
      }
      // (the stage is not filled again before it was waited for here)
      if (lane == 0) tc::bar_arrive(&sh.k_free[st]);
    }
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
  }
}

template <int DP, bool BF16, class Sh>
__device__ __forceinline__ void issue_role(const GradParams& p, Sh& sh, uint32_t q_smem, uint32_t do_smem, uint32_t k_smem, uint32_t v_smem,
                                           uint32_t tmem, int t) {
  using S = Shape<DP>;
  constexpr uint32_t id_s = tc::idesc16(BF16, 128, kKeys, false), id_o = tc::idesc16(BF16, 128, DP, true);
  const uint64_t kmajor = tc::sdesc_sw128(0), mnmajor = tc::sdesc_mn_sw128(0, kKeys * kRowBytes);
  const uint32_t km = tc::desc_hi(kmajor), mn = tc::desc_hi(mnmajor);
  const uint32_t dq = (uint32_t)kmajor + ((q_smem + t * S::kTile) >> 4), ddo = (uint32_t)kmajor + ((do_smem + t * S::kTile) >> 4);
  const uint32_t dk = (uint32_t)kmajor + (k_smem >> 4), dv = (uint32_t)kmajor + (v_smem >> 4), dkt = (uint32_t)mnmajor + (k_smem >> 4);
  const uint32_t s_at = tmem + t * 256, dp_at = s_at + 64, o_at = s_at + 128;
  uint32_t j = 0, done = 0, n_q = 0, n_o = 0;
  uint32_t looked = 0;  // a bit a stage: how often (mod 2) its keys were looked at
  struct {
    bool any, mine, first, last;
  } was = {false, false, false, false};
  uint32_t i = 0;
  int k = 0, steps = 0, nk = 0, whole = 0;  // whole: steps that end before the keys do
  for (;;) {
    if (k == steps) {
      if (i > 0) tc::bar_arrive(&sh.item_free[(i - 1) % kItems]);
      WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
      steps = sh.item[i % kItems].steps;
      nk = steps == 0 ? 0 : sh.item[i % kItems].nk[t];
      whole = sh.item[i % kItems].keys / kKeys;
      k = 0;
      ++i;
    }
    const bool end = steps == 0, mine = !end && k < nk;
    const uint32_t st = j % S::kStagesK, sv = j % S::kStagesV, before = (j - 1) % S::kStagesK;
    if (!end) {
      WAIT(sh.k_full[st], (j / S::kStagesK) & 1);
      if (k >= whole) {
        WAIT(sh.k_ready[st], (looked >> st) & 1);
        looked ^= 1u << st;
      }
    }
    if (mine) {
      if (k == 0) {
        WAIT(sh.q_full[t], n_q & 1);
        ++n_q;
      }
      if (done > 0) WAIT(sh.s_read[t], (done - 1) & 1);
      tc::fence_after();
#pragma unroll
      for (int q = 0; q < DP / 16; ++q)
        tc::mma16_ss(s_at, dq + (q >> 2) * (128 * kRowBytes >> 4) + (q & 3) * 2, km,
                     dk + st * (S::kHalf >> 4) + (q >> 2) * (kKeys * kRowBytes >> 4) + (q & 3) * 2, km, id_s, q > 0);
      tc::mma_commit(&sh.s_full[t]);
    }
    if (was.any) {
      if (was.mine) {
        if (was.first) {
          WAIT(sh.o_free[t], (n_o & 1) ^ 1);
          ++n_o;
        }
        WAIT(sh.ds_full[t], (done - 1) & 1);
        tc::fence_after();
#pragma unroll
        for (int q = 0; q < kKeys / 16; ++q)
          tc::mma16_ts(o_at, dp_at + q * 8, dkt + before * (S::kHalf >> 4) + q * (16 * kRowBytes >> 4), mn, id_o, q > 0 || !was.first);
        if (was.last) tc::mma_commit(&sh.o_full[t]);
      }
      was.mine ? tc::mma_commit(&sh.k_free[before]) : tc::bar_arrive(&sh.k_free[before]);
    }
    if (end) return;
    WAIT(sh.v_full[sv], (j / S::kStagesV) & 1);
    if (mine) {
      tc::fence_after();
#pragma unroll
      for (int q = 0; q < DP / 16; ++q)
        tc::mma16_ss(dp_at, ddo + (q >> 2) * (128 * kRowBytes >> 4) + (q & 3) * 2, km,
                     dv + sv * (S::kHalf >> 4) + (q >> 2) * (kKeys * kRowBytes >> 4) + (q & 3) * 2, km, id_s, q > 0);
      tc::mma_commit(&sh.dp_full[t]);
      tc::mma_commit(&sh.v_free[sv]);
      if (k == nk - 1) tc::mma_commit(&sh.q_free[t]);
    } else {
      tc::bar_arrive(&sh.v_free[sv]);
    }
    was.any = true;
    was.mine = mine;
    was.first = k == 0;
    was.last = k == nk - 1;
    if (mine) ++done;
    ++j;
    ++k;
  }
}

// A row a thread
template <int DP, bool BF16, class Sh>
__device__ __forceinline__ void element_role(const GradParams& p, Sh& sh, uint32_t tmem, int t) {
  const int r = threadIdx.x & 127, lane = threadIdx.x & 31;
  const uint32_t s_at = tmem + t * 256 + ((uint32_t)(r & ~31) << 16), dp_at = s_at + 64;
  const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
  uint32_t done = 0;
  for (uint32_t i = 0;; ++i) {
    WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
    const PromptItem& x = sh.item[i % kItems];
    const int steps = x.steps, nk = x.nk[t], rows = x.rows, keys = x.keys;
    if (steps == 0) return;
    const int first = (x.tile * 2 + t) << (7 - p.log2P), tok = first + (r >> p.log2P), head0 = x.hb << p.log2P;
    const int64_t row0 = x.row0, at = (row0 + tok) * p.H + head0 + (r & ((1 << p.log2P) - 1));
    __syncwarp();
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
    if (nk == 0) continue;
    const int limit = min(prompt_limit(p, rows, keys, tok), keys), common = min(prompt_limit(p, rows, keys, first), keys);
    float2 stat = make_float2(INFINITY, 0.f);
    if (tok < rows && in_bounds(at < p.total_rows * p.H, p.status, kSitePromptRow)) stat = p.stat[at];
    const float power = BF16 ? 1.f : p.power[row0 * p.Hkv + head0 / p.G];
    const float2 add2 = make_float2(-stat.x, -stat.x), delta2 = make_float2(stat.y * power, stat.y * power);
    const float2 power2 = make_float2(power, power);
#pragma unroll 1
    for (int k = 0; k < nk; ++k, ++done) {
      WAIT(sh.s_full[t], done & 1);
      tc::fence_after();
      // (32 columns at a time: 64 at once need registers that are not there)
      float pr[64];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t v[32];
        tc::tmem_ld32(s_at + 32 * c, v);
        tc::wait_ld(v);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float2 y = tc::fma2(make_float2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), scale2, add2);
          pr[32 * c + 2 * e] = fast_exp2(y.x);
          pr[32 * c + 2 * e + 1] = fast_exp2(y.y);
        }
        if (c == 1) {
          tc::fence_before();
          tc::bar_arrive(&sh.s_read[t]);
        }
      }
      if (PROMPT_RARE((k + 1) * kKeys > common)) {
        const int lim = (limit == 1 ? 0 : limit) - k * kKeys;  // (a row that sees one key: dS is 0, as in the kernel of keys)
#pragma unroll
        for (int e = 0; e < 64; ++e) pr[e] = e < lim ? pr[e] : 0.f;
      }
      WAIT(sh.dp_full[t], done & 1);
      tc::fence_after();
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t v[32];
        tc::tmem_ld32(dp_at + 32 * c, v);
        tc::wait_ld(v);
        // keys past the end: what is there may be anything
        if (PROMPT_RARE(k * kKeys + kKeys > keys)) {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = k * kKeys + 32 * c + e < keys ? v[e] : 0u;
        }
        uint32_t pk[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float2 y = tc::fma2(make_float2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), power2, delta2);
          y = tc::mul2(y, make_float2(pr[32 * c + 2 * e], pr[32 * c + 2 * e + 1]));
          pk[e] = pack16<BF16>(y.x, y.y);
        }
        tc::tmem_st16(dp_at + 16 * c, pk);
      }
      tc::tmem_wait_st();
      tc::fence_before();
      tc::bar_arrive(&sh.ds_full[t]);
    }
  }
}

template <int DP, bool BF16, class Sh>
__device__ __forceinline__ void write_role(const GradParams& p, Sh& sh, unsigned char* stage, uint32_t tmem) {
  const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31;
  const uint32_t lanes = (uint32_t)(warp * 32) << 16;
  const RowWriter writer{stage + warp * (32 * 128), lane};
  uint32_t n[2] = {0, 0};
  for (uint32_t i = 0;; ++i) {
    WAIT(sh.item_full[i % kItems], (i / kItems) & 1);
    const PromptItem x = sh.item[i % kItems];
    if (x.steps == 0) return;
    const float f = BF16 ? p.scale : p.scale / p.power[x.row0 * p.Hkv + (x.hb << p.log2P) / p.G];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (x.nk[t] == 0) continue;
      WAIT(sh.o_full[t], n[t] & 1);
      tc::fence_after();
      ++n[t];
#pragma unroll 1
      for (int blk = 0; blk < Shape<DP>::kBlocks; ++blk) {
        const int cols = min(DP - blk * 64, 64);
#pragma unroll 1
        for (int c = 0; c < cols; c += 16) {
          uint32_t o[16], w[8];
          tc::tmem_ld16(tmem + t * 256 + 128 + lanes + blk * 64 + c, o);
          scale_pack<BF16>(o, f, w);
          writer.put16(c, w);
        }
        if (blk == Shape<DP>::kBlocks - 1) {
          tc::fence_before();
          tc::bar_arrive(&sh.o_free[t]);
        }
        writer.flush(blk, p.dim / 8, [&](int rr) -> uint16_t* {
          const int row = warp * 32 + rr, tok = ((x.tile * 2 + t) << (7 - p.log2P)) + (row >> p.log2P);
          return tok < x.rows && in_bounds(x.row0 + tok < p.total_rows, p.status, kSitePromptRow)
                     ? p.dq + (x.row0 + tok) * p.dq_row + ((x.hb << p.log2P) + (row & ((1 << p.log2P) - 1))) * p.dim
                     : nullptr;
        });
      }
    }
    __syncwarp();
    if (lane == 0) tc::bar_arrive(&sh.item_free[i % kItems]);
  }
}

template <int DP, bool BF16>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_rows_kernel(GradParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_do,
                       const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using S = Shape<DP>;
  using Sh = Shared<S::kStagesK, S::kStagesV>;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* q_smem = smem;
  unsigned char* do_smem = q_smem + 2 * S::kTile;
  unsigned char* k_smem = do_smem + 2 * S::kTile;
  unsigned char* v_smem = k_smem + S::kStagesK * S::kHalf;
  unsigned char* stage = v_smem + S::kStagesV * S::kHalf;
  Sh& sh = *reinterpret_cast<Sh*>(stage + 4 * 32 * 128);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    sh.stop = 0;
    for (int k = 0; k < 2; ++k) {
      tc::bar_init(&sh.q_full[k], 1);
      tc::bar_init(&sh.q_free[k], 1);
      tc::bar_init(&sh.s_full[k], 1);
      tc::bar_init(&sh.s_read[k], 128);
      tc::bar_init(&sh.dp_full[k], 1);
      tc::bar_init(&sh.ds_full[k], 128);
      tc::bar_init(&sh.o_full[k], 1);
      tc::bar_init(&sh.o_free[k], 128);
    }
    for (int k = 0; k < S::kStagesK; ++k) {
      tc::bar_init(&sh.k_full[k], 1);
      tc::bar_init(&sh.k_ready[k], 1);
      tc::bar_init(&sh.k_free[k], 3);
    }
    for (int k = 0; k < S::kStagesV; ++k) {
      tc::bar_init(&sh.v_full[k], 1);
      tc::bar_init(&sh.v_free[k], 2);
    }
    for (int k = 0; k < kItems; ++k) {
      tc::bar_init(&sh.item_full[k], 1);
      tc::bar_init(&sh.item_free[k], 16);  // every warp
    }
    tc::bar_init(&sh.drain, 2);
    tc::bar_fence_init();
  }
  pdl_wait();
  if (warp == 12) tc::tmem_alloc(&sh.tmem, 512);
  prompt_list(p, sh.list, Count{p}, p.most);
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  const uint32_t tmem = sh.tmem;
  if (warp < 8) {
    tc::setmaxnreg_inc<kRegElement>();
    element_role<DP, BF16>(p, sh, tmem, warp >> 2);
  } else if (warp < 12) {
    tc::setmaxnreg_dec<kRegWrite>();
    write_role<DP, BF16>(p, sh, stage, tmem);
  } else {
    tc::setmaxnreg_dec<kRegIssue>();
    if (warp == 13)
      load_role<DP>(p, sh, map_q, map_do, map_k, map_v, q_smem, do_smem, k_smem, v_smem);
    else if (warp == 15)
      look_role<DP>(p, sh, k_smem);
    else if (tc::elect_one())
      issue_role<DP, BF16>(p, sh, tc::su32(q_smem), tc::su32(do_smem), tc::su32(k_smem), tc::su32(v_smem), tmem, warp == 14);
  }
  __syncthreads();
  // after a wait that ran out, products and copies may still be in flight
  if (sh.stop && (warp == 12 || warp == 14) && tc::elect_one()) {
    tc::mma_commit(&sh.drain);
    tc::bar_wait(&sh.drain, 0, nullptr, kPromptWaitNs);
    for (int k = 0; k < 2 * (S::kStagesK + S::kStagesV + 2); ++k) {
      const int n = k / 2 - S::kStagesK;
      uint64_t* bar = n < 0 ? &sh.k_full[k / 2] : n < S::kStagesV ? &sh.v_full[n] : &sh.q_full[n - S::kStagesV];
      tc::bar_wait(bar, k & 1, nullptr, kPromptWaitNs / 16);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) prompt_leave(p, gridDim.x, sh.stop);
  if (warp == 12) tc::tmem_dealloc(tmem, 512);
}

}  // namespace rows

// dV and dK of the items that were divided: their parts' sums in order. A CTA takes 32 keys of a tile: grid x over the
// sequences' tiles, found as the kernel of keys finds its items (offsets may go back behind a sequence that does not
// fit), y over key heads and the two gradients, z over quarters.
struct Tiles {
  __device__ __forceinline__ int operator()(const PromptSeq& s) const { return s.keys / 128 + (s.keys % 128 != 0); }
};
template <bool BF16>
__global__ void __launch_bounds__(256) split_kernel(GradParams p, int log_p) {
  __shared__ PromptList list;
  __shared__ PromptSeq sh_seq;
  __shared__ int sh_tile;
  pdl_wait();
  prompt_list(p, list, Tiles{}, p.most_keys / (p.Hkv * p.parts));
  if ((int)blockIdx.x >= list.first[kChunks]) return;
  if (threadIdx.x < 32) {
    PromptTaker at;
    at.find(p, list, Tiles{}, blockIdx.x);
    if (threadIdx.x == 0) {
      sh_seq = at.s;
      sh_tile = (int)blockIdx.x - at.begin;
    }
  }
  __syncthreads();
  const PromptSeq s = sh_seq;
  const int64_t first = (int64_t)sh_tile * 128 + blockIdx.z * 32;
  if (first >= s.keys) return;
  const keys::Tile x(p, s, sh_tile, log_p);
  if (x.parts < 2) return;
  const int hb = blockIdx.y >> 1, which = blockIdx.y & 1, pieces = p.dim / 4, keys = (int)min((int64_t)32, s.keys - first);
  uint16_t* base = which ? p.dk : p.dv;
  const int64_t row = which ? p.dk_row : p.dv_row, part = 2 * p.total_keys * p.Hkv * p.dim;
  for (int e = threadIdx.x; e < keys * pieces; e += 256) {
    const int r = e / pieces, c = (e - r * pieces) * 4;
    const int64_t key = s.key0 + first + r;
    if (!in_bounds(key < p.total_keys, p.status, kSitePromptRow)) continue;
    const float* from = p.split + ((which * p.total_keys + key) * p.Hkv + hb) * p.dim + c;
    float4 y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = k < x.parts ? *reinterpret_cast<const float4*>(from + k * part) : make_float4(0.f, 0.f, 0.f, 0.f);
    float4 sum = y[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) {
      sum.x += y[k].x;
      sum.y += y[k].y;
      sum.z += y[k].z;
      sum.w += y[k].w;
    }
    *reinterpret_cast<uint2*>(base + key * row + hb * p.dim + c) = make_uint2(pack16<BF16>(sum.x, sum.y), pack16<BF16>(sum.z, sum.w));
  }
}

// Once per device and kernel: the shared memory, and that the register split adds up --
// setmaxnreg.inc waits for registers that only the launch's own can give.
template <class Kernel, class... Maps>
int launch(Kernel kern, std::atomic<uint64_t>& ready, int smem, int grid, cudaStream_t st, const GradParams& p, const Maps&... maps) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return OCCAM_ERR_CUDA;
  if (!((ready.load(std::memory_order_acquire) >> dev) & 1)) {
    cudaFuncAttributes at;
    if (cudaFuncGetAttributes(&at, kern) != cudaSuccess) return OCCAM_ERR_CUDA;
    if (at.numRegs * kThreads < 256 * kRegElement + 128 * (kRegWrite + kRegIssue)) return OCCAM_ERR_UNSUPPORTED;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return OCCAM_ERR_CUDA;
    ready.fetch_or(uint64_t(1) << dev, std::memory_order_release);
  }
  return launch_after(kern, dim3((unsigned)grid), kThreads, smem, st, p, maps...) && cudaGetLastError() == cudaSuccess
             ? OCCAM_OK
             : OCCAM_ERR_CUDA;
}

template <int DP, bool BF16>
int launch_grad(const GradParams& p, const CUtensorMap (&mk)[5], const CUtensorMap (&mr)[4], int grid_keys, int grid_rows, cudaStream_t st) {
  if (p.total_rows > 0) {
    const int log_lanes = p.dim <= 64 ? 3 : 4;
    const int64_t most = std::max(p.total_rows * p.H, BF16 ? 0 : p.total_keys * p.Hkv), per = (256 >> log_lanes) * kVectors;
    if ((most + per - 1) / per > 0x7fffffff) return OCCAM_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((most + per - 1) / per), BF16 ? 1 : 2);
    if (!(log_lanes == 3 ? launch_after(stat_kernel<BF16, 3>, grid, 256, 0, st, p) : launch_after(stat_kernel<BF16, 4>, grid, 256, 0, st, p)))
      return OCCAM_ERR_CUDA;
    if (!BF16 && !launch_after(power_kernel, dim3((unsigned)p.n, (unsigned)p.Hkv), 512, 0, st, p)) return OCCAM_ERR_CUDA;
  }
  using K = keys::Shape<DP>;
  using R = rows::Shape<DP>;
  constexpr int smem_k = (2 + K::kStages) * K::kTile + 4 * 32 * 128 + 2 * keys::kUnitBytes + K::kStages * keys::kMoreBytes +
                         (int)sizeof(keys::Shared<K::kStages>);
  constexpr int smem_r =
      4 * R::kTile + (R::kStagesK + R::kStagesV) * R::kHalf + 4 * 32 * 128 + (int)sizeof(rows::Shared<R::kStagesK, R::kStagesV>);
  static_assert(smem_k <= 227 * 1024 && smem_r <= 227 * 1024, "an SM's shared memory");
  static std::atomic<uint64_t> ready_k{0}, ready_r{0};
  if (grid_keys > 0) {
    const int rc = launch(keys::prompt_keys_kernel<DP, BF16>, ready_k, smem_k, grid_keys, st, p, mk[0], mk[1], mk[2], mk[3], mk[4]);
    if (rc != OCCAM_OK) return rc;
  }
  if (grid_rows > 0) {
    const int rc = launch(rows::prompt_rows_kernel<DP, BF16>, ready_r, smem_r, grid_rows, st, p, mr[0], mr[1], mr[2], mr[3]);
    if (rc != OCCAM_OK) return rc;
  }
  if (p.parts > 1 && grid_keys > 0) {
    const dim3 grid((unsigned)(p.most_keys / (p.Hkv * p.parts)), (unsigned)p.Hkv * 2, 4);
    if (!launch_after(split_kernel<BF16>, grid, 256, 0, st, p, std::min(p.log2P, 6)) || cudaGetLastError() != cudaSuccess) return OCCAM_ERR_CUDA;
  }
  return OCCAM_OK;
}

}  // namespace

#define OCCAM_TRY(x)                 \
  do {                               \
    int _rc = (x);                   \
    if (_rc != OCCAM_OK) return _rc; \
  } while (0)

extern "C" int occam_prompt_attend_grad(const occam_prompt_args* a, const occam_prompt_grads* g, void* workspace, size_t workspace_bytes,
                                        occam_stream_t stream) {
  const NvtxRange nvtx("occam_prompt_attend_grad");
  launch_counter() = 0;
  GradParams p{};
  OCCAM_TRY(prompt_params(a, workspace, workspace_bytes, &p));
  if (!g) return OCCAM_ERR_INVALID_ARG;
  const PromptWs w = prompt_ws(a->total_rows, a->total_keys, a->heads, a->kv_heads);
  if (workspace_bytes < w.total) return OCCAM_ERR_WORKSPACE;
  if (a->n == 0 || (a->total_rows == 0 && a->total_keys == 0)) return OCCAM_OK;
  const int64_t R = a->total_rows, K = a->total_keys, qw = (int64_t)a->heads * a->dim, kw = (int64_t)a->kv_heads * a->dim;
  auto fits = [&](const void* x, int64_t rows, int64_t row, int64_t width) {
    return rows == 0 || (x && aligned16(x) && (row & 7) == 0 && row >= width && row < (int64_t(1) << 38));
  };
  if (!fits(g->out, R, qw, qw) || (R > 0 && !g->lse) || !fits(g->dout, R, g->dout_row, qw) || !fits(g->dq, R, g->dq_row, qw) ||
      !fits(g->dk, K, g->dk_row, kw) || !fits(g->dv, K, g->dv_row, kw))
    return OCCAM_ERR_INVALID_ARG;
  // no result lies over an input or over another result
  const Extent to[3] = {extent(g->dq, R, g->dq_row, 1, 0, qw, 2), extent(g->dk, K, g->dk_row, 1, 0, kw, 2),
                        extent(g->dv, K, g->dv_row, 1, 0, kw, 2)};
  const bool there[3] = {R > 0, K > 0, K > 0};
  for (int i = 0; i < 3; ++i) {
    if (!there[i]) continue;
    if (prompt_meets_inputs(a, to[i])) return OCCAM_ERR_INVALID_ARG;
    if (R > 0 && (meet(to[i], extent(g->out, R, qw, 1, 0, qw, 2)) || meet(to[i], extent(g->dout, R, g->dout_row, 1, 0, qw, 2)) ||
                  meet(to[i], extent(g->lse, 1, 0, 1, 0, R * a->heads * 2, 2))))
      return OCCAM_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (there[j] && meet(to[i], to[j])) return OCCAM_ERR_INVALID_ARG;
  }
  p.o = static_cast<const uint16_t*>(g->out);
  p.lse = const_cast<float*>(g->lse);
  p.dout = static_cast<const uint16_t*>(g->dout);
  p.dout_row = g->dout_row;
  p.v = static_cast<const uint16_t*>(a->v);
  p.v_row = a->v_row;
  p.dq = static_cast<uint16_t*>(g->dq);
  p.dk = static_cast<uint16_t*>(g->dk);
  p.dv = static_cast<uint16_t*>(g->dv);
  p.dq_row = g->dq_row;
  p.dk_row = g->dk_row;
  p.dv_row = g->dv_row;
  p.stat = ws_at<float2>(workspace, w.stat);
  p.terms = ws_at<uint4>(workspace, w.terms);
  p.norm = ws_at<float>(workspace, w.norm);
  p.vnorm = ws_at<float>(workspace, w.vnorm);
  p.power = ws_at<float>(workspace, w.power);
  const bool bf16 = a->dtype == OCCAM_BF16;
  const int per = 256 >> p.log2P, heads = p.H >> p.log2P, log_p = std::min(p.log2P, 6);
  const int64_t most_rows = R == 0 ? 0 : (R / per + a->n) * heads, most_keys = K == 0 ? 0 : (K / 128 + a->n) * p.Hkv;
  if (most_rows > (1 << 30) || most_keys > (1 << 30) || (!bf16 && p.Hkv > 65535)) return OCCAM_ERR_UNSUPPORTED;
  // Few items of keys are divided, where one may have the steps for it: a group's heads by blocks of 64 rows.
  p.parts = prompt_parts(std::max<int64_t>((K + 127) / 128, a->n) * p.Hkv);
  if ((R / (64 >> log_p) + 1) * (p.G >> log_p) < 2 * keys::kPartSteps) p.parts = 1;
  p.split = ws_at<float>(workspace, w.split);
  p.most = (int)most_rows;
  p.most_keys = (int)(most_keys * p.parts);
  // (without any rows, or any keys, the copies have to come from somewhere; what they bring is not used)
  const void* q = R > 0 ? a->q : a->k;
  const void* dout = R > 0 ? g->dout : a->k;
  const void* k = K > 0 ? a->k : a->q;
  const void* v = K > 0 ? a->v : a->q;
  const int64_t q_row = R > 0 ? a->q_row : (int64_t(1) << 20), do_row = R > 0 ? g->dout_row : (int64_t(1) << 20);
  const int64_t k_row = K > 0 ? a->k_row : a->q_row, v_row = K > 0 ? a->v_row : a->q_row;
  const int64_t rows = std::max<int64_t>(R, 1), keys_n = std::max<int64_t>(K, 1);
  CUtensorMap mk[5], mr[4];
  if (!encode_rows(&mk[0], q, bf16, p.dim, p.H, rows, q_row, 1 << log_p, 64 >> log_p) ||
      !encode_rows(&mk[1], dout, bf16, p.dim, p.H, rows, do_row, 1 << log_p, 64 >> log_p) ||
      !encode_rows(&mk[2], k, bf16, p.dim, p.Hkv, keys_n, k_row, 1, 128) || !encode_rows(&mk[3], v, bf16, p.dim, p.Hkv, keys_n, v_row, 1, 128) ||
      !encode_rows(&mk[4], p.terms, bf16, 16, p.H, rows, 16 * (int64_t)p.H, 1 << log_p, 64 >> log_p, 16) ||
      !encode_rows(&mr[0], q, bf16, p.dim, p.H, rows, q_row, 1 << p.log2P, 128 >> p.log2P) ||
      !encode_rows(&mr[1], dout, bf16, p.dim, p.H, rows, do_row, 1 << p.log2P, 128 >> p.log2P) ||
      !encode_rows(&mr[2], k, bf16, p.dim, p.Hkv, keys_n, k_row, 1, 64) || !encode_rows(&mr[3], v, bf16, p.dim, p.Hkv, keys_n, v_row, 1, 64))
    return OCCAM_ERR_CUDA;
  const int grid_rows = (int)std::min<int64_t>(cache_sms(), most_rows), grid_keys = (int)std::min<int64_t>(cache_sms(), p.most_keys);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (p.dim <= 64)
    return bf16 ? launch_grad<64, true>(p, mk, mr, grid_keys, grid_rows, st) : launch_grad<64, false>(p, mk, mr, grid_keys, grid_rows, st);
  if (p.dim <= 80)
    return bf16 ? launch_grad<80, true>(p, mk, mr, grid_keys, grid_rows, st) : launch_grad<80, false>(p, mk, mr, grid_keys, grid_rows, st);
  return bf16 ? launch_grad<128, true>(p, mk, mr, grid_keys, grid_rows, st) : launch_grad<128, false>(p, mk, mr, grid_keys, grid_rows, st);
}
