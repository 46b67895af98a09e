// Attention over the paged 8-bit cache for many query rows (prompts, long chunks), on
// the 5th-generation tensor cores.  The mathematics is that of pq_kv8_rows.
//
// Split.  A block takes one cache head and 256 query rows (queries x heads of the group)
// as two tiles of 128, and walks through the tokens 128 at a time.  Each step's codes
// are turned into halves once, for both tiles, on their way into shared memory.  The
// softmax works on half a step: scores are 128 rows x 64 tokens in tensor memory, a row
// a thread, so it needs no exchange between threads; the probabilities go back over the
// scores as halves and are the second product's first operand from there.  Each tile has
// two such buffers: the next half's scores are computed while this one's softmax runs
// (with one buffer of 128 tokens the softmax waited for its own product and the next scores,
// 4600 cycles a step).  One thread's MMAs run in order, so scores never overwrite
// probabilities in use.  The outputs stay in tensor memory; they are rescaled only when
// a row's maximum has grown by more than 2^8 (w, scaled by 2^6, stays below 2^14; a half holds 2^16).
// Bound by waiting: at D = 128 a step's products take 2560 cycles (scores of 64 tokens wait for
// shared memory, 48 cycles an MMA instead of 32), a step about 4900 over a whole launch, and no pipe is near its limit (issue 53 %,
// tensor 40 %, exponentials 20 %).  Both tiles share their barriers, so their softmax runs at one time and little covers it; a warp and
// barriers for each tile, with eight or six converting warps, cost more (a window of 2048 and 16 sinks, two prompts of 4096 over 10000: 284 us, so
// 340 and 393).  Four prompts of 2048 over 4096, 32 / 8 heads of 128: 249 us.
//
// Roles (16 warps): 0 issues the MMAs, 4 looks up pages, the other six below 8 convert
// (none of them on the issuing warp's scheduler), 8-11 and 12-15 are the tiles' softmax.  One tile of rows has other roles, and 20 warps
// (TcRoles).  Tiles with the most tokens come first.
#pragma once

#include <cuda_runtime.h>

#include <type_traits>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_kv8.cuh"
#include "pq_tokens.cuh"

namespace pq {
namespace {

constexpr int kTokens = kAttnTcTokens;  // of one step
constexpr int kHalf = 64;               // of one round of the softmax
constexpr int kSub = 128 * 128;         // 128 rows of 64 halves
constexpr int kPageRing = 8;            // steps whose pages are looked up ahead

// Queries of two tiles (wide: of one), two stages of keys and values as halves, wide: two steps' codes.
__host__ __device__ constexpr int attn_smem(int DP, bool wide) {
  return (wide ? 5 : 6) * (DP / 64) * kSub + (wide ? 2 * 2 * kTokens * DP : 0) + 1024 /* alignment */;
}

struct AttnBars {
  uint32_t base;
  __device__ uint32_t q_full() const { return base; }
  __device__ uint32_t done() const { return base + 8u; }
  __device__ uint32_t k_full(int s) const { return base + 16u + 8u * s; }
  __device__ uint32_t k_empty(int s) const { return base + 32u + 8u * s; }
  __device__ uint32_t v_full(int s) const { return base + 48u + 8u * s; }
  __device__ uint32_t v_empty(int s) const { return base + 64u + 8u * s; }
  // scores and probabilities in buffer b (of both tiles, 2; of the two streams, 4), outputs (of both tiles; of stream t)
  __device__ uint32_t s_full(int b) const { return base + 80u + 8u * b; }
  __device__ uint32_t p_full(int b) const { return base + 112u + 8u * b; }
  __device__ uint32_t o_full(int t) const { return base + 144u + 8u * t; }
  __device__ uint32_t page_full(int i) const { return base + 160u + 8u * i; }
  __device__ uint32_t page_empty(int i) const { return base + 160u + 8u * kPageRing + 8u * i; }
};
constexpr int kBars = 20 + 2 * kPageRing;

// A page of a step: scale of the keys, log2 and inverse of the values' scale, and where
// the head's codes begin (absent pages: -1).
struct alignas(8) StepPage {
  float k, log2_v, inv_v;
  int64_t codes;
};

// Operand descriptors in two words.  Both in the 128-byte swizzle, groups of 8 rows 1024
// bytes apart.  K-major: rows of 64 halves of K.  N-major: rows are K (tokens), their 64-wide
// column blocks (of D) kSub apart.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_k(uint32_t addr) { return ((addr >> 4) & 0x3FFFu) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_n(uint32_t addr) { return ((addr >> 4) & 0x3FFFu) | (static_cast<uint32_t>(kSub >> 4) << 16); }

// Four MMAs (64 of K); the whole warp calls, one lane issues.  One election and no
// branch between them: a branch around each made the issue of an MMA take longer than
// the MMA.  The first operand from shared memory (32 bytes of K a step) or tensor memory.
__device__ __forceinline__ void mma_ss_x4(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p, q, e;\n.reg .b64 x, y;\nelect.sync _|e, 0xffffffff;\nsetp.ne.b32 p, %10, 0;\nsetp.eq.b32 q, 0, 0;\n"
      "mov.b64 x, {%1, %11};\nmov.b64 y, {%5, %11};\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %9, p;\n"
      "mov.b64 x, {%2, %11};\nmov.b64 y, {%6, %11};\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %9, q;\n"
      "mov.b64 x, {%3, %11};\nmov.b64 y, {%7, %11};\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %9, q;\n"
      "mov.b64 x, {%4, %11};\nmov.b64 y, {%8, %11};\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %9, q;\n}" ::"r"(d),
      "r"(a), "r"(a + 2), "r"(a + 4), "r"(a + 6), "r"(b), "r"(b + 2), "r"(b + 4), "r"(b + 6), "r"(idesc), "r"(accumulate),
      "r"(kDescHigh)
      : "memory");
}
// (16 rows of the second operand, 2048 bytes, a step)
__device__ __forceinline__ void mma_ts_x4(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p, q, e;\n.reg .b64 y;\nelect.sync _|e, 0xffffffff;\nsetp.ne.b32 p, %10, 0;\nsetp.eq.b32 q, 0, 0;\n"
      "mov.b64 y, {%5, %11};\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %9, p;\n"
      "mov.b64 y, {%6, %11};\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%2], y, %9, q;\n"
      "mov.b64 y, {%7, %11};\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%3], y, %9, q;\n"
      "mov.b64 y, {%8, %11};\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%4], y, %9, q;\n}" ::"r"(d),
      "r"(a), "r"(a + 8), "r"(a + 16), "r"(a + 24), "r"(b), "r"(b + 128), "r"(b + 256), "r"(b + 384), "r"(idesc),
      "r"(accumulate), "r"(kDescHigh)
      : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// (s0, s1) += (a, b), packed.
__device__ __forceinline__ void add_pair(float& s0, float& s1, float a, float b) {
  asm("{\n.reg .b64 s, t;\nmov.b64 s, {%0, %1};\nmov.b64 t, {%2, %3};\nadd.rn.f32x2 s, s, t;\nmov.b64 {%0, %1}, s;\n}"
      : "+f"(s0), "+f"(s1)
      : "f"(a), "f"(b));
}

// Where the block works: the row tile is the slowest part, the last ones (which see
// the most tokens) first.
struct TcPlace {
  int tile, split, h, b;
};
__device__ __forceinline__ TcPlace tc_place(const AttnArgs& p) {
  TcPlace r;
  unsigned i = blockIdx.x;
  r.h = i % p.c.Hkv;
  i /= p.c.Hkv;
  r.split = i % p.splits;
  i /= p.splits;
  r.b = i % p.a.B;
  r.tile = p.row_tiles - 1 - static_cast<int>(i / p.a.B);
  return r;
}

// How the warps share the work.  Two tiles of rows: six converting warps beside the issuing one and the pages', off the issuing
// warp's scheduler, and four of softmax for each tile.  Wide, for one tile of rows: the two groups of softmax are streams of the same
// rows, one through the first half of every step and one through the second, with maxima, sums and outputs of their own, joined at
// the end (one group had 1100 to 1900 cycles' work with each half, and everything else waited for it); each stream has a warp of
// its own that issues its MMAs (one warp needed 3600 cycles for both streams' 24 MMAs, 6 waits and 7 commits of a step, and
// everything else waited for it: 32 sequences of up to 24 drafts over up to 6000 103.9 us, so 94.8); four warps convert the keys and
// four the values.  Bound by the softmax now: 2000 to 2200 of a step's 2800 cycles for 64 tokens of a row, and about 400 of hand-over.
template <bool WIDE>
struct TcRoles {
  static constexpr int kThreads = WIDE ? 640 : 512;
  static constexpr int kOneSide = WIDE ? 4 : 6;  // converting warps of the keys (and of the values)
  static constexpr int kPageWarp = WIDE ? 1 : 4, kSecondIssuer = 2, kFirstConverter = 4, kFirstSoftmax = WIDE ? 12 : 8;
  // this warp's number among the converting ones
  static __device__ __forceinline__ int converter(int warp) { return WIDE ? warp - kFirstConverter : warp < 4 ? warp - 1 : warp - 2; }
};

// VIEW: see AttnView.
template <typename T, int DP, int VIEW, bool WIDE>
__global__ void __launch_bounds__(TcRoles<WIDE>::kThreads, 1) pq_kv8_tiles(const __grid_constant__ AttnArgs p) {
  using Roles = TcRoles<WIDE>;
  constexpr int kSubs = DP / 64;
  constexpr uint32_t kO = 256;  // tensor memory: scores of both tiles, then their outputs
  extern __shared__ uint8_t raw[];
  __shared__ alignas(8) uint64_t bar_words[kBars];
  __shared__ StepPage pages[kPageRing][8];
  __shared__ int abort_flag;
  __shared__ uint32_t tmem_base;
  TcPlace w = tc_place(p);
  if (WIDE && p.in_order) w.b = longest_first(p, w.b, reinterpret_cast<int*>(raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r0 = w.tile * kAttnTcRows;
  const Span sp = span_of(p, w.b, r0, kAttnTcRows);
  const int rows = sp.n * p.group;
  if (r0 >= rows) return;
  // (with sinks, steps are counted without the gap behind them; token() has it)
  const Walk walk = walk_of(p, sp);
  const int from = (VIEW == kSinks ? 0 : walk.gap) + w.split * p.chunk;
  const int end = VIEW == kSinks ? walk.end : sp.hi;
  if (w.split > 0 && from >= end) return;
  const int to = min(end, from + p.chunk);
  auto token = [&](int s) { return VIEW == kSinks && s >= walk.head ? s + walk.gap : s; };
  const int steps = to > from ? (to - from + kTokens - 1) / kTokens : 0;
  const int halves = to > from ? (to - from + kHalf - 1) / kHalf : 0;
  const int streams = WIDE || rows - r0 > 128 ? 2 : 1;  // of MMAs and softmax: the tiles with rows, wide: both halves of a step
  const int D = p.c.D;
  const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t q_base = smem, k_base = q_base + (WIDE ? 1 : 2) * kSubs * kSub, v_base = k_base + 2 * kSubs * kSub;
  const AttnBars bars{smem_u32(bar_words)};

  if (threadIdx.x == 0) {
    mbar_init(bars.q_full(), 4 * streams);
    mbar_init(bars.done(), WIDE ? streams : 1);
    for (int s = 0; s < 2; ++s) {
      mbar_init(bars.k_full(s), Roles::kOneSide);
      mbar_init(bars.k_empty(s), WIDE ? streams : 1);
      mbar_init(bars.v_full(s), Roles::kOneSide);
      mbar_init(bars.v_empty(s), WIDE ? streams : 1);
    }
    for (int b = 0; b < 4; ++b) {
      mbar_init(bars.s_full(b), 1);
      mbar_init(bars.p_full(b), 4 * (WIDE ? 1 : streams));
    }
    for (int b = 0; b < 2; ++b) mbar_init(bars.o_full(b), 1);
    for (int i = 0; i < kPageRing; ++i) {
      mbar_init(bars.page_full(i), 1);
      mbar_init(bars.page_empty(i), 1);
    }
    abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 0) tmem_alloc(smem_u32(&tmem_base), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // all 512 columns are this block's: the base is 0 (a constant address costs the issuing
  // warp no register moves)
  constexpr uint32_t tmem = 0;
  WaitCtx ctx{&abort_flag, p.err, p.wait_limit_ns, PQ_ERR_MMA};

  auto finish = [&]() {
    // every MMA issued is over: the outputs are whole, the tensor memory may be given back
    tc_commit_warp(bars.done());
    if (lane == 0) mbar_wait_drain(bars.done(), 0, p.wait_limit_ns, p.err);
    __syncwarp();
  };
  auto issue_both = [&]() {
    // ---- MMAs of both tiles
    auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, ctx)) != 0; };
    const uint32_t idesc_s = (1u << 4) | (8u << 17) | (8u << 24);                                        // N = 64 tokens
    const uint32_t idesc_o = (1u << 4) | (1u << 16) | (static_cast<uint32_t>(D >> 3) << 17) | (8u << 24);  // N = D
    // Half i is half i % 2 of step i / 2, whose operands are in stage (i / 2) % 2.  Both
    // tiles share barriers: a wait or a commit costs this warp about as much as two MMAs.
    auto scores = [&](int i) {
      const uint32_t k = k_base + ((i >> 1) & 1) * kSubs * kSub + (i & 1) * (kHalf * 128);
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (t < streams) {
#pragma unroll
          for (int c = 0; c < kSubs; ++c)
            mma_ss_x4(tmem + 128 * t + kHalf * (i & 1), desc_k(q_base + (t * kSubs + c) * kSub), desc_k(k + c * kSub),
                      idesc_s, c > 0);
        }
      tc_commit_warp(bars.s_full(i & 1));
    };
    auto outputs = [&](int i) {
      const uint32_t v = desc_n(v_base + ((i >> 1) & 1) * kSubs * kSub + (i & 1) * (kHalf * 128));
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (t < streams) {
          mma_ts_x4(tmem + kO + t * DP, tmem + 128 * t + kHalf * (i & 1), v, idesc_o, i > 0);
          if (kSecondHalf<T, VIEW>) mma_ts_x4(tmem + kO + t * DP, tmem + 128 * t + kHalf * (i & 1) + kHalf / 2, v, idesc_o, 1);
        }
      tc_commit_warp(bars.o_full(0));
    };
    bool ok = halves > 0 && wait(bars.q_full(), 0) && wait(bars.k_full(0), 0);
    if (ok) {
      tc_fence_after();
      scores(0);
    }
    for (int i = 0; ok && i < halves; ++i) {
      const int j = i >> 1, n = i + 1;
      if (n < halves) {
        if (!(n & 1)) ok = wait(bars.k_full((n >> 1) & 1), (n >> 2) & 1);
        if (!ok) break;
        tc_fence_after();
        scores(n);
      }
      if (!(i & 1)) {  // both halves of the step's keys have been issued
        tc_commit_warp(bars.k_empty(j & 1));
        ok = wait(bars.v_full(j & 1), (j >> 1) & 1);
      }
      ok = ok && wait(bars.p_full(i & 1), j & 1);
      if (!ok) break;
      tc_fence_after();
      outputs(i);
      if ((i & 1) || n == halves) tc_commit_warp(bars.v_empty(j & 1));
    }
    finish();
  };
  // ---- wide: MMAs of stream t, which takes half t of every step (its `turn`)
  auto issue = [&](auto which) {
    constexpr int t = decltype(which)::value;
    const int turns = (halves + 1 - t) >> 1;
    auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, ctx)) != 0; };
    const uint32_t idesc_s = (1u << 4) | (8u << 17) | (8u << 24);                                        // N = 64 tokens
    const uint32_t idesc_o = (1u << 4) | (1u << 16) | (static_cast<uint32_t>(D >> 3) << 17) | (8u << 24);  // N = D
    auto scores = [&](int turn) {
      const int s = turn & 1;
      const uint32_t k = k_base + s * kSubs * kSub + t * (kHalf * 128);
#pragma unroll
      for (int c = 0; c < kSubs; ++c)
        mma_ss_x4(tmem + 128 * t + kHalf * s, desc_k(q_base + c * kSub), desc_k(k + c * kSub), idesc_s, c > 0);
      tc_commit_warp(bars.s_full(2 * t + s));
      tc_commit_warp(bars.k_empty(s));
    };
    auto outputs = [&](int turn) {
      const int s = turn & 1;
      const uint32_t v = desc_n(v_base + s * kSubs * kSub + t * (kHalf * 128)), weights = tmem + 128 * t + kHalf * s;
      mma_ts_x4(tmem + kO + t * DP, weights, v, idesc_o, turn > 0);
      if (kSecondHalf<T, VIEW>) mma_ts_x4(tmem + kO + t * DP, weights + kHalf / 2, v, idesc_o, 1);
      tc_commit_warp(bars.o_full(t));
      tc_commit_warp(bars.v_empty(s));
    };
    bool ok = turns > 0 && wait(bars.q_full(), 0) && wait(bars.k_full(0), 0);
    if (ok) {
      tc_fence_after();
      scores(0);
    }
    for (int turn = 0; ok && turn < turns; ++turn) {
      const int next = turn + 1;
      if (next < turns) {
        ok = wait(bars.k_full(next & 1), (next >> 1) & 1);
        if (!ok) break;
        tc_fence_after();
        scores(next);
      }
      ok = wait(bars.v_full(turn & 1), (turn >> 1) & 1) && wait(bars.p_full(2 * t + (turn & 1)), (turn >> 1) & 1);
      if (!ok) break;
      tc_fence_after();
      outputs(turn);
    }
    finish();
  };
  auto look_up = [&]() {
    // ---- the steps' pages, a lane each, up to kPageRing steps ahead of the codes (two
    // dependent loads that would otherwise stand in every step's way)
    ctx.err_bits = PQ_ERR_PRODUCER;
    const int* table = p.a.page_table_dev + static_cast<int64_t>(w.b) * p.a.table_pitch;
    for (int j = 0; j < steps; ++j) {
      const int i = j % kPageRing;
      if (j >= kPageRing &&
          !__all_sync(0xffffffffu, mbar_wait(bars.page_empty(i), (j / kPageRing - 1) & 1, ctx)))
        break;
      if (lane < kTokens >> p.page_shift) {
        const int start = token(from + j * kTokens) + (lane << p.page_shift), slot = start >> p.page_shift;
        StepPage page = {0.0f, kNone, 0.0f, -1};
        if (start < sp.hi && (start + p.c.page_tokens > sp.lo || (VIEW == kSinks && start < p.sinks))) {  // within the rows' span
          const int id = slot < p.a.table_pitch ? table[slot] : -1;
          if (id >= 0 && id < p.c.num_pages) {
            const int64_t ph = static_cast<int64_t>(id) * p.c.Hkv + w.h;
            const float sk = p.c.k_scale_dev[ph], sv0 = p.c.v_scale_dev[ph], sv = sv0 == 0.0f ? kZeroPageScale : sv0;
            page = {sk, log2f(sv), 1.0f / sv, (ph << p.page_shift) * D};
          } else {
            atomicOr(p.err, PQ_ERR_PAGE);
          }
        }
        pages[i][lane] = page;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bars.page_full(i));
    }
  };
  auto convert = [&]() {
    // ---- codes to halves
    ctx.err_bits = PQ_ERR_PRODUCER;
    const int side = WIDE && Roles::converter(warp) >= Roles::kOneSide;  // wide: keys or values
    const int tid = 32 * (Roles::converter(warp) - side * Roles::kOneSide) + lane;
    const int C = D / 16;  // 16-byte pieces of a token
    // A thread takes one 16-byte piece of every kTokStep-th token.  Eight neighbours
    // hold four pieces of two tokens, whose halves lie in different banks.
    constexpr int kP = DP / 16, kTokStep = 32 * Roles::kOneSide / kP, kTurns = (kTokens + kTokStep - 1) / kTokStep;
    const int piece = kP == 8 ? (tid & 3) | ((tid >> 1) & 4) : tid & 3;
    const int token = kP == 8 ? ((tid >> 3) & ~1) | ((tid >> 2) & 1) : tid >> 2;
    const bool there = piece < C;
    const uint32_t row = (piece >> 2) * kSub + token * 128;
    const uint32_t at0 = row + (((2 * (piece & 3)) ^ (token & 7)) << 4), at1 = row + (((2 * (piece & 3) + 1) ^ (token & 7)) << 4);
    // every step's pieces lie at the same places of its pages
    auto slot = [&](int i) { return (WIDE ? token + i * kTokStep : min(token + i * kTokStep, kTokens - 1)) >> p.page_shift; };
    auto in_page = [&](int i) { return ((token + i * kTokStep) & (p.c.page_tokens - 1)) * D + 16 * piece; };
    // wide: a step's codes are on their way through shared memory two steps ahead (each thread copies what it will convert; one step ahead
    // in registers, half of a step's time went by waiting for them); else through registers
    const uint32_t staged = v_base + 2 * kSubs * kSub + tid * 16;
    auto copy = [&](const int8_t* codes, int j) {
      if (j < steps) {
        const StepPage* page = pages[j % kPageRing];
        // (all looked up before the first copy: in turn, eight of them took 1900 cycles)
        int64_t bases[kTurns];
#pragma unroll
        for (int i = 0; i < kTurns; ++i) bases[i] = page[slot(i)].codes;
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
          const int64_t base = bases[i];
          const bool have = base >= 0 && there;
          cp_async_16(staged + ((j & 1) * 2 + side) * (kTokens * DP) + i * (32 * Roles::kOneSide * 16), have ? codes + base + in_page(i) : codes,
                      have ? 16 : 0);
        }
      }
      cp_async_commit();
    };
    static_assert(!WIDE || kTurns * kTokStep == kTokens, "every turn is whole");
    constexpr int kBatch = kTurns < 4 ? kTurns : 4;  // turns at a time
    auto arrived = [&](int j, int i0, uint4 (&r)[kBatch]) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[i].x), "=r"(r[i].y), "=r"(r[i].z), "=r"(r[i].w)
                     : "r"(staged + ((j & 1) * 2 + side) * (kTokens * DP) + (i0 + i) * (32 * Roles::kOneSide * 16))
                     : "memory");
    };
    auto fetch = [&](const int8_t* codes, int j, uint4 (&r)[kTurns]) {
      const StepPage* page = pages[j % kPageRing];
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int64_t base = page[slot(i)].codes;
        r[i] = make_uint4(0, 0, 0, 0);
        if (base >= 0 && there && token + i * kTokStep < kTokens) r[i] = *reinterpret_cast<const uint4*>(codes + base + in_page(i));
      }
    };
    // (columns past D are zeros: the scores' products run over whole blocks of 64)
    auto store = [&](uint32_t base, const uint4* r, int n) {
#pragma unroll
      for (int i = 0; i < n; ++i) {
        if (!WIDE && token + i * kTokStep >= kTokens) break;
        uint32_t h[8];
        half_of_codes(r[i].x, h[0], h[1]);
        half_of_codes(r[i].y, h[2], h[3]);
        half_of_codes(r[i].z, h[4], h[5]);
        half_of_codes(r[i].w, h[6], h[7]);
        sts128(base + at0 + i * kTokStep * 128, h[0], h[1], h[2], h[3]);
        sts128(base + at1 + i * kTokStep * 128, h[4], h[5], h[6], h[7]);
      }
    };
    auto publish = [&](uint32_t bar) {
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    auto look = [&](int j) {
      return __all_sync(0xffffffffu, mbar_wait(bars.page_full(j % kPageRing), (j / kPageRing) & 1, ctx)) != 0;
    };
    if constexpr (WIDE) {
      const int8_t* codes = side ? p.c.v_dev : p.c.k_dev;
      const uint32_t base = side ? v_base : k_base, full = side ? bars.v_full(0) : bars.k_full(0), empty = side ? bars.v_empty(0) : bars.k_empty(0);
      bool ok = true;
      for (int j = 0; ok && j < 2; ++j) {
        if (j < steps) ok = look(j);
        if (ok) copy(codes, j);
      }
      for (int j = 0; ok && j < steps; ++j) {
        const int s = j & 1;
        if (j > 1) ok = __all_sync(0xffffffffu, mbar_wait(empty + 8u * s, ((j >> 1) - 1) & 1, ctx)) != 0;
        if (!ok) break;
        // values: step j - 2 is over, and so is every use of its pages
        if (j > 1 && side && tid == 0) mbar_arrive(bars.page_empty((j - 2) % kPageRing));
        cp_async_wait<1>();
#pragma unroll
        for (int i = 0; i < kTurns; i += kBatch) {
          uint4 r[kBatch];
          arrived(j, i, r);
          store(base + s * kSubs * kSub + i * kTokStep * 128, r, kBatch);
        }
        publish(full + 8u * s);
        if (j + 2 < steps) ok = look(j + 2);
        if (ok) copy(codes, j + 2);
      }
      cp_async_wait<0>();
      return;
    }
    uint4 kr[kTurns], vr[kTurns];
    bool ok = steps > 0 && look(0);
    if (ok) {
      fetch(p.c.k_dev, 0, kr);
      fetch(p.c.v_dev, 0, vr);
    }
    for (int j = 0; ok && j < steps; ++j) {
      const int s = j & 1;
      if (j > 1) ok = __all_sync(0xffffffffu, mbar_wait(bars.k_empty(s), ((j >> 1) - 1) & 1, ctx)) != 0;
      if (!ok) break;
      store(k_base + s * kSubs * kSub, kr, kTurns);
      publish(bars.k_full(s));
      if (j + 1 < steps) {
        ok = look(j + 1);
        if (!ok) break;
        fetch(p.c.k_dev, j + 1, kr);
      }
      if (j > 1) ok = __all_sync(0xffffffffu, mbar_wait(bars.v_empty(s), ((j >> 1) - 1) & 1, ctx)) != 0;
      if (!ok) break;
      // step j - 2 is over: so is every use of its pages
      if (j > 1 && tid == 0) mbar_arrive(bars.page_empty((j - 2) % kPageRing));
      store(v_base + s * kSubs * kSub, vr, kTurns);
      publish(bars.v_full(s));
      if (j + 1 < steps) fetch(p.c.v_dev, j + 1, vr);
    }
  };

  // (the registers of all together are what the threads had at launch: 512 of 128, 640 of 96)
  if (!WIDE && warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    if (warp == 0)
      issue_both();
    else if (warp == Roles::kPageWarp)
      look_up();
    else
      convert();
  } else if (WIDE && warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == 0)
      issue(std::integral_constant<int, 0>{});
    else if (warp == Roles::kPageWarp)
      look_up();
    else if (warp == Roles::kSecondIssuer)
      issue(std::integral_constant<int, 1>{});
  } else if (WIDE && warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    convert();
  } else {
    if (WIDE)
      asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
    else
      asm volatile("setmaxnreg.inc.sync.aligned.u32 152;");
    // ---- softmax: this thread's row
    ctx.err_bits = PQ_ERR_EPILOGUE;
    const int t = (warp - Roles::kFirstSoftmax) >> 2;
    if (t < streams) {
      const int in = 32 * (warp & 3) + lane, r = r0 + (WIDE ? 0 : 128 * t) + in;
      const bool mine = r < rows;
      const int qi = mine ? r / p.group : 0, hq = w.h * p.group + (mine ? r % p.group : 0);
      const int64_t tok = static_cast<int64_t>(p.a.cu_q_dev[w.b]) + qi;
      const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16;
      const uint32_t s_mem = tmem + lanes + 128 * t, o_mem = tmem + lanes + kO + t * DP;
      float factor;
      {
        // the row as halves, scaled so that its largest element lies in [2^7, 2^8)
        const T* src = static_cast<const T*>(p.q) + tok * p.a.q_token_stride + static_cast<int64_t>(hq) * p.a.q_head_stride;
        Vec8<T> v[DP / 8];
        uint32_t top = 0;
        // (all of a row's loads on their way at one time: with a branch around each they took 9000 cycles, one after the other.  Rows past
        // the end read the sequence's first and count as zeros.)
        if (p.wide_q) {
#pragma unroll
          for (int i = 0; i < DP / 8; ++i) v[i] = load8(src + (8 * i < D ? 8 * i : 0), 8, true);
#pragma unroll
          for (int i = 0; i < DP / 8; ++i)
            if (!mine || 8 * i >= D) v[i] = Vec8<T>{};
        } else {
#pragma unroll
          for (int i = 0; i < DP / 8; ++i) v[i] = load8(src + 8 * i, mine && 8 * i < D ? 8 : 0, false);
        }
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) top = max(top, amax8(v[i]));
        const int e = top >= 0x7F800000u ? 0 : max(static_cast<int>(top >> 23) - 127, -100);
        // (negated where the call's scale is negative: the scores' factor is not)
        const float f = __int_as_float((127 + 7 - e) << 23) * (p.a.scale < 0.0f ? -1.0f : 1.0f);
        factor = fabsf(p.a.scale) * kLog2e * __int_as_float((127 - 7 + e) << 23);
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) {
          if (WIDE && i / (DP / 16) != t) continue;  // (each stream's threads write half of the row)
          uint32_t h[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) h[k] = pack_half2(to_f32(v[i].v[2 * k]) * f, to_f32(v[i].v[2 * k + 1]) * f);
          sts128(q_base + ((WIDE ? 0 : t * kSubs) + i / 8) * kSub + in * 128 + (((i & 7) ^ (in & 7)) << 4), h[0], h[1], h[2], h[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bars.q_full());
      }
      const int at = sp.len - sp.n + qi + 1;
      // (rows past the end see everything, so that their warp's others need no masks; nothing of theirs is written)
      const int hi = !mine ? (VIEW == kPlain ? 0 : 0x7FFFFFFF) : p.a.causal ? min(at, sp.len) : sp.len;
      const int lo = p.a.window > 0 && (mine || VIEW == kPlain) ? max(0, at - p.a.window) : 0;
      // the draft's row of bits (one that is there for rows past the end), and the first draft's position
      const uint32_t* drafts = VIEW == kTree ? p.tree + (mine ? tok : p.a.cu_q_dev[w.b]) * p.tree_pitch : nullptr;
      const int text = sp.len - sp.n;
      float m = kNone, l = 0.0f;
      bool ok = true;
      int i = WIDE ? t : 0;
      if (WIDE && __all_sync(0xffffffffu, !mine)) {  // a warp whose rows are all past the end only keeps the barriers' count
        for (; ok && i < halves; i += 2) {
          const int turn = i >> 1, place = 2 * t + (turn & 1);
          ok = __all_sync(0xffffffffu, mbar_wait(bars.s_full(place), (turn >> 1) & 1, ctx)) != 0;
          if (lane == 0 && ok) mbar_arrive(bars.p_full(place));
        }
      }
      for (; i < halves; i += WIDE ? 2 : 1) {
        const int turn = WIDE ? i >> 1 : i, place = WIDE ? 2 * t + (turn & 1) : turn & 1;  // of this group's halves; its buffer's barriers
        ok = __all_sync(0xffffffffu, mbar_wait(bars.s_full(place), (turn >> 1) & 1, ctx)) != 0;
        if (!ok) break;
        tc_fence_after();
        const uint32_t buffer = s_mem + kHalf * (turn & 1);
        float x[kHalf];
#pragma unroll
        for (int c = 0; c < kHalf; c += 32) {
          uint32_t v[32];
          tmem_ld32(buffer + c, v);
#pragma unroll
          for (int k = 0; k < 32; ++k) x[c + k] = __uint_as_float(v[k]);
        }
        tmem_wait_ld();
        const StepPage* page = pages[(i >> 1) % kPageRing];
        const int c0 = kHalf * (i & 1), j0 = token(from + i * kHalf);
        const bool whole = __all_sync(0xffffffffu, (j0 >= lo || (VIEW == kSinks && j0 + kHalf <= p.sinks)) &&
                                                       j0 + kHalf <= (VIEW == kTree && mine ? min(hi, text) : hi)) != 0;
        // the row's maximum: within 16 tokens of one page that of the raw scores (the scales
        // are not negative)
        float high = m;
        if (whole) {
#pragma unroll
          for (int c = 0; c < kHalf; c += 16) {
            const StepPage& f = page[(c0 + c) >> p.page_shift];
            float top = fmaxf(x[c], x[c + 1]);
#pragma unroll
            for (int k = 2; k < 16; k += 2) top = fmaxf(top, fmaxf(x[c + k], x[c + k + 1]));
            high = fmaxf(high, fmaf(top, f.k * factor, f.log2_v));
          }
        } else {
          uint32_t bits[2] = {};
          if (VIEW == kTree) {
            bits[0] = first_bits(hi - j0) & drafts_seen(drafts, p.tree_words, j0 - text);
            bits[1] = first_bits(hi - j0 - 32) & drafts_seen(drafts, p.tree_words, j0 + 32 - text);
          }
          if (VIEW == kSinks) {
            bits[0] = first_bits(hi - j0) & (~first_bits(lo - j0) | first_bits(p.sinks - j0));
            bits[1] = first_bits(hi - j0 - 32) & (~first_bits(lo - j0 - 32) | first_bits(p.sinks - j0 - 32));
          }
#pragma unroll
          for (int c = 0; c < kHalf; c += 16) {
            const StepPage& f = page[(c0 + c) >> p.page_shift];
            const float g = f.k * factor, lv = f.log2_v;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const bool seen = VIEW == kPlain ? j0 + c + k >= lo && j0 + c + k < hi : ((bits[c / 32] >> ((c & 16) + k)) & 1u) != 0;
              x[c + k] = seen ? fmaf(x[c + k], g, lv) : kNone;
              high = fmaxf(high, x[c + k]);
            }
          }
        }
        const bool grew = high > m + kGrow;
        if (__any_sync(0xffffffffu, grew)) {
          const float next = grew ? high : m;
          const float alpha = next == kNone ? 1.0f : exp2_approx(m - next);
          m = next;
          l *= alpha;
          if (turn > 0) {
            // once the product of the half before is over
            ok = __all_sync(0xffffffffu, mbar_wait(bars.o_full(WIDE ? t : 0), (turn - 1) & 1, ctx)) != 0;
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < DP; c += 16) {
              if (c < D) {
                uint32_t v[16];
                tmem_ld16(o_mem + c, v);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * alpha);
                tmem_st16(o_mem + c, v);
              }
            }
          }
        }
        const float base = m == kNone ? 0.0f : m - kWShift;
#pragma unroll
        for (int c = 0; c < kHalf; c += 32) {
          uint32_t h[16], rest[kSecondHalf<T, VIEW> ? 16 : 1];
#pragma unroll
          for (int u = 0; u < 32; u += 16) {
            const StepPage& f = page[(c0 + c + u) >> p.page_shift];
            // seen as a whole: the scores are still raw
            const float g = whole ? f.k * factor : 1.0f, shift = whole ? f.log2_v - base : -base;
            float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
              float a, b;
              fma2_rn(x[c + u + k], x[c + u + k + 1], g, shift, a, b);
              a = exp2_approx(a);
              b = exp2_approx(b);
              add_pair(s0, s1, a, b);
              if (kSecondHalf<T, VIEW>) {
                // 11 bits by truncation: what is left is exact
                const float a1 = __uint_as_float(__float_as_uint(a) & 0xFFFFE000u), b1 = __uint_as_float(__float_as_uint(b) & 0xFFFFE000u);
                rest[kSecondHalf<T, VIEW> ? (u + k) / 2 : 0] = pack_half2(a - a1, b - b1);
                a = a1;
                b = b1;
              }
              h[(u + k) / 2] = pack_half2(a, b);
            }
            // a page that the row does not see adds nothing, even with a NaN scale
            const float sum = s0 + s1;
            l += whole || sum != 0.0f ? sum * f.inv_v : 0.0f;
          }
          tmem_st16(buffer + c / 2, h);
          if constexpr (kSecondHalf<T, VIEW>) tmem_st16(buffer + kHalf / 2 + c / 2, rest);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bars.p_full(place));
      }
      // ---- outputs
      if (ok && steps > 0) ok = __all_sync(0xffffffffu, mbar_wait(bars.done(), 0, ctx)) != 0;
      tc_fence_after();
      float weight[2] = {1.0f, 0.0f};  // wide: of each stream's outputs
      // (without a step nothing has waited for the other warps' queries to be written, and there is nothing to join: every row has none)
      if (WIDE && steps > 0) {
        // the streams' maxima and sums, in the queries' place
        float2 (*joined)[128] = reinterpret_cast<float2 (*)[128]>(raw + (q_base - smem_u32(raw)));
        joined[t][in] = make_float2(m, l);
        asm volatile("bar.sync 1, 256;" ::: "memory");
        const float2 a = joined[0][in], b = joined[1][in];
        m = fmaxf(a.x, b.x);
        const float top = m == kNone ? 0.0f : m;
        weight[0] = exp2_approx(a.x - top), weight[1] = exp2_approx(b.x - top);
        l = a.y * weight[0] + b.y * weight[1];
      }
      const float inv = p.splits > 1 ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
      const int64_t part = ((static_cast<int64_t>(w.b) * p.a.max_q + qi) * p.a.Hq + hq) * p.splits + w.split;
      if (p.splits > 1 && mine && (!WIDE || t == 0)) p.ml[part] = make_float2(m, l);
      T* dst = static_cast<T*>(p.o) + tok * p.a.o_token_stride + static_cast<int64_t>(hq) * p.a.o_head_stride;
#pragma unroll
      for (int c = 0; c < DP; c += 16) {
        if (WIDE && c / (DP / 2) != t) continue;  // (each stream's threads write half of the row)
        if (c < D) {
          uint32_t v[16];
          if constexpr (WIDE) {
            uint32_t u[16];
            tmem_ld16(tmem + lanes + kO + c, v);
            tmem_ld16(tmem + lanes + kO + DP + c, u);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              // (the second stream has written nothing where there is one half)
              const float second = halves > 1 ? __uint_as_float(u[i]) * weight[1] : 0.0f;
              v[i] = __float_as_uint(fmaf(__uint_as_float(v[i]), weight[0], second));
            }
          } else {
            tmem_ld16(o_mem + c, v);
            tmem_wait_ld();
          }
          if (!ok || !mine) continue;
          if (p.splits > 1) {
#pragma unroll
            for (int i = 0; i < 16; i += 2)
              *reinterpret_cast<float2*>(p.part + part * D + c + i) =
                  steps > 0 ? make_float2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])) : make_float2(0.0f, 0.0f);
          } else {
#pragma unroll
            for (int u = 0; u < 16; u += 8) {
              Vec8<T> r;
#pragma unroll
              for (int i = 0; i < 8; ++i)
                r.v[i] = from_f32<T>(steps > 0 && l != 0.0f ? __uint_as_float(v[u + i]) * inv : 0.0f);
              store8(dst + c + u, r, 8, p.wide_o);
            }
          }
        }
      }
      tc_fence_before();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

template <typename T, int DP, int VIEW, bool WIDE>
cudaError_t launch_tiles_as(const AttnArgs& p, unsigned grid, cudaStream_t stream) {
  static int attr_set[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(pq_kv8_tiles<T, DP, VIEW, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, attn_smem(DP, WIDE));
    if (e != cudaSuccess) return e;
    if (dev < 64) attr_set[dev] = 1;
  }
  pq_kv8_tiles<T, DP, VIEW, WIDE><<<grid, TcRoles<WIDE>::kThreads, attn_smem(DP, WIDE), stream>>>(p);
  return cudaGetLastError();
}

template <typename T, int DP, int VIEW>
cudaError_t launch_tiles(const AttnArgs& p, unsigned grid, cudaStream_t stream) {
  if constexpr (VIEW != kPlain)  // (its order of sums is another than the one that plain attention has always had)
    if (static_cast<int64_t>(p.a.max_q) * p.group <= 128) return launch_tiles_as<T, DP, VIEW, true>(p, grid, stream);
  return launch_tiles_as<T, DP, VIEW, false>(p, grid, stream);
}

}  // namespace

template <int VIEW>
cudaError_t launch_attn_tc(const AttnArgs& p, unsigned grid, cudaStream_t stream) {
  if (p.a.type == PQ_F16) return p.c.D <= 64 ? launch_tiles<__half, 64, VIEW>(p, grid, stream) : launch_tiles<__half, 128, VIEW>(p, grid, stream);
  return p.c.D <= 64 ? launch_tiles<__nv_bfloat16, 64, VIEW>(p, grid, stream) : launch_tiles<__nv_bfloat16, 128, VIEW>(p, grid, stream);
}

}  // namespace pq
