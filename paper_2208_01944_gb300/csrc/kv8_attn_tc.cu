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
// shared memory, 48 cycles an MMA instead of 32), a step about 5500 over a whole launch, and no pipe is near its limit (issue 48 %,
// exponentials 19 %).  Both tiles share their barriers, so their softmax runs at one time and little covers it.  Four prompts
// of 2048 over 4096, 32 / 8 heads of 128: 278 us (0.79 PFLOP/s); one of 8192, causal: 569 us (0.97 PFLOP/s).
//
// Roles (16 warps): 0 issues the MMAs, 4 looks up pages, the other six below 8 convert
// (none of them on the issuing warp's scheduler), 8-11 and 12-15 are the tiles' softmax.  Tiles with the most tokens come first.
#include <cuda_runtime.h>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_kv8.cuh"
#include "pq_tokens.cuh"

namespace pq {
namespace {

constexpr int kTokens = kAttnTcTokens;  // of one step
constexpr int kHalf = 64;               // of one round of the softmax
constexpr int kThreads = 512;
constexpr int kSub = 128 * 128;         // 128 rows of 64 halves
constexpr int kPageRing = 8;            // steps whose pages are looked up ahead

__host__ __device__ constexpr int attn_smem(int DP) { return 6 * (DP / 64) * kSub + 1024 /* alignment */; }

struct AttnBars {
  uint32_t base;
  __device__ uint32_t q_full() const { return base; }
  __device__ uint32_t done() const { return base + 8u; }
  __device__ uint32_t k_full(int s) const { return base + 16u + 8u * s; }
  __device__ uint32_t k_empty(int s) const { return base + 32u + 8u * s; }
  __device__ uint32_t v_full(int s) const { return base + 48u + 8u * s; }
  __device__ uint32_t v_empty(int s) const { return base + 64u + 8u * s; }
  // both tiles' scores and probabilities in buffer b; their outputs
  __device__ uint32_t s_full(int b) const { return base + 80u + 8u * b; }
  __device__ uint32_t p_full(int b) const { return base + 96u + 8u * b; }
  __device__ uint32_t o_full() const { return base + 112u; }
  __device__ uint32_t page_full(int i) const { return base + 120u + 8u * i; }
  __device__ uint32_t page_empty(int i) const { return base + 120u + 8u * kPageRing + 8u * i; }
};
constexpr int kBars = 15 + 2 * kPageRing;

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

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, 1) pq_kv8_tiles(const __grid_constant__ AttnArgs p) {
  constexpr int kSubs = DP / 64;
  constexpr uint32_t kO = 256;  // tensor memory: scores of both tiles, then their outputs
  extern __shared__ uint8_t raw[];
  __shared__ alignas(8) uint64_t bar_words[kBars];
  __shared__ StepPage pages[kPageRing][8];
  __shared__ int abort_flag;
  __shared__ uint32_t tmem_base;
  const TcPlace w = tc_place(p);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r0 = w.tile * kAttnTcRows;
  const Span sp = span_of(p, w.b, r0, kAttnTcRows);
  const int rows = sp.n * p.group;
  if (r0 >= rows) return;
  const int first = sp.lo & ~(p.align - 1);
  const int from = first + w.split * p.chunk;
  if (w.split > 0 && from >= sp.hi) return;
  const int to = min(sp.hi, from + p.chunk);
  const int steps = to > from ? (to - from + kTokens - 1) / kTokens : 0;
  const int halves = to > from ? (to - from + kHalf - 1) / kHalf : 0;
  const int tiles = rows - r0 > 128 ? 2 : 1;
  const int D = p.c.D;
  const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t q_base = smem, k_base = q_base + 2 * kSubs * kSub, v_base = k_base + 2 * kSubs * kSub;
  const AttnBars bars{smem_u32(bar_words)};

  if (threadIdx.x == 0) {
    mbar_init(bars.q_full(), 4 * tiles);
    mbar_init(bars.done(), 1);
    for (int s = 0; s < 2; ++s) {
      mbar_init(bars.k_full(s), 6);
      mbar_init(bars.k_empty(s), 1);
      mbar_init(bars.v_full(s), 6);
      mbar_init(bars.v_empty(s), 1);
      mbar_init(bars.s_full(s), 1);
      mbar_init(bars.p_full(s), 4 * tiles);
    }
    mbar_init(bars.o_full(), 1);
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

  if (warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    if (warp == 0) {
      // ---- MMAs
      auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, ctx)) != 0; };
      const uint32_t idesc_s = (1u << 4) | (8u << 17) | (8u << 24);                                        // N = 64 tokens
      const uint32_t idesc_o = (1u << 4) | (1u << 16) | (static_cast<uint32_t>(D >> 3) << 17) | (8u << 24);  // N = D
      // Half i is half i % 2 of step i / 2, whose operands are in stage (i / 2) % 2.  Both
      // tiles share barriers: a wait or a commit costs this warp about as much as two MMAs.
      auto scores = [&](int i) {
        const uint32_t k = k_base + ((i >> 1) & 1) * kSubs * kSub + (i & 1) * (kHalf * 128);
#pragma unroll
        for (int t = 0; t < 2; ++t)
          if (t < tiles) {
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
          if (t < tiles) mma_ts_x4(tmem + kO + t * DP, tmem + 128 * t + kHalf * (i & 1), v, idesc_o, i > 0);
        tc_commit_warp(bars.o_full());
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
      // every MMA issued is over: the outputs are whole, the tensor memory may be given back
      tc_commit_warp(bars.done());
      if (lane == 0) mbar_wait_drain(bars.done(), 0, p.wait_limit_ns, p.err);
      __syncwarp();
    } else if (warp == 4) {
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
          const int start = from + j * kTokens + (lane << p.page_shift), slot = start >> p.page_shift;
          StepPage page = {0.0f, kNone, 0.0f, -1};
          if (start < sp.hi && start + p.c.page_tokens > sp.lo) {  // within the rows' span
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
    } else {
      // ---- codes to halves, six warps
      ctx.err_bits = PQ_ERR_PRODUCER;
      const int tid = 32 * (warp < 4 ? warp - 1 : warp - 2) + lane;
      const int C = D / 16;  // 16-byte pieces of a token
      // A thread takes one 16-byte piece of every (192 / kP)th token.  Eight neighbours
      // hold four pieces of two tokens, whose halves lie in different banks.
      constexpr int kP = DP / 16, kTokStep = 192 / kP, kTurns = (kTokens + kTokStep - 1) / kTokStep;
      const int piece = kP == 8 ? (tid & 3) | ((tid >> 1) & 4) : tid & 3;
      const int token = kP == 8 ? ((tid >> 3) & ~1) | ((tid >> 2) & 1) : tid >> 2;
      const bool there = piece < C;
      const uint32_t row = (piece >> 2) * kSub + token * 128;
      const uint32_t at0 = row + (((2 * (piece & 3)) ^ (token & 7)) << 4), at1 = row + (((2 * (piece & 3) + 1) ^ (token & 7)) << 4);
      auto fetch = [&](const int8_t* codes, int j, uint4 (&r)[kTurns]) {
        const StepPage* page = pages[j % kPageRing];
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
          const int k = token + i * kTokStep;
          r[i] = make_uint4(0, 0, 0, 0);
          if (!there || k >= kTokens) continue;
          const int64_t base = page[k >> p.page_shift].codes;
          if (base >= 0)
            r[i] = *reinterpret_cast<const uint4*>(codes + base + (k & (p.c.page_tokens - 1)) * D + 16 * piece);
        }
      };
      // (columns past D are zeros: the scores' products run over whole blocks of 64)
      auto store = [&](uint32_t base, const uint4 (&r)[kTurns]) {
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
          if (token + i * kTokStep >= kTokens) break;
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
        store(k_base + s * kSubs * kSub, kr);
        publish(bars.k_full(s));
        if (j + 1 < steps) {
          ok = look(j + 1);
          if (!ok) break;
          fetch(p.c.k_dev, j + 1, kr);
        }
        if (j > 1) ok = __all_sync(0xffffffffu, mbar_wait(bars.v_empty(s), ((j >> 1) - 1) & 1, ctx)) != 0;
        if (!ok) break;
        // step j - 2 is over: so is every use of its pages
        if (j > 1 && warp == 1 && lane == 0) mbar_arrive(bars.page_empty((j - 2) % kPageRing));
        store(v_base + s * kSubs * kSub, vr);
        publish(bars.v_full(s));
        if (j + 1 < steps) fetch(p.c.v_dev, j + 1, vr);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 152;");
    // ---- softmax: this thread's row
    ctx.err_bits = PQ_ERR_EPILOGUE;
    const int t = (warp - 8) >> 2;
    if (t < tiles) {
      const int in = 32 * (warp & 3) + lane, r = r0 + 128 * t + in;
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
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) {
          const bool there = mine && 8 * i < D;
          v[i] = load8(src + 8 * i, there ? 8 : 0, there && p.wide_q);
          top = max(top, amax8(v[i]));
        }
        const int e = top >= 0x7F800000u ? 0 : max(static_cast<int>(top >> 23) - 127, -100);
        // (negated where the call's scale is negative: the scores' factor is not)
        const float f = __int_as_float((127 + 7 - e) << 23) * (p.a.scale < 0.0f ? -1.0f : 1.0f);
        factor = fabsf(p.a.scale) * kLog2e * __int_as_float((127 - 7 + e) << 23);
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) {
          uint32_t h[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) h[k] = pack_half2(to_f32(v[i].v[2 * k]) * f, to_f32(v[i].v[2 * k + 1]) * f);
          sts128(q_base + (t * kSubs + i / 8) * kSub + in * 128 + (((i & 7) ^ (in & 7)) << 4), h[0], h[1], h[2], h[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bars.q_full());
      }
      const int at = sp.len - sp.n + qi + 1;
      const int hi = !mine ? 0 : p.a.causal ? min(at, sp.len) : sp.len;
      const int lo = p.a.window > 0 ? max(0, at - p.a.window) : 0;
      float m = kNone, l = 0.0f;
      bool ok = true;
      for (int i = 0; i < halves; ++i) {
        ok = __all_sync(0xffffffffu, mbar_wait(bars.s_full(i & 1), (i >> 1) & 1, ctx)) != 0;
        if (!ok) break;
        tc_fence_after();
        const uint32_t buffer = s_mem + kHalf * (i & 1);
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
        const int c0 = kHalf * (i & 1), j0 = from + i * kHalf;
        const bool whole = __all_sync(0xffffffffu, j0 >= lo && j0 + kHalf <= hi) != 0;
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
#pragma unroll
          for (int c = 0; c < kHalf; c += 16) {
            const StepPage& f = page[(c0 + c) >> p.page_shift];
            const float g = f.k * factor, lv = f.log2_v;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const bool seen = j0 + c + k >= lo && j0 + c + k < hi;
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
          if (i > 0) {
            // once the product of the half before is over
            ok = __all_sync(0xffffffffu, mbar_wait(bars.o_full(), (i - 1) & 1, ctx)) != 0;
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
          uint32_t h[16];
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
              h[(u + k) / 2] = pack_half2(a, b);
            }
            // a page that the row does not see adds nothing, even with a NaN scale
            const float sum = s0 + s1;
            l += whole || sum != 0.0f ? sum * f.inv_v : 0.0f;
          }
          tmem_st16(buffer + c / 2, h);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bars.p_full(i & 1));
      }
      // ---- outputs
      if (ok && steps > 0) ok = __all_sync(0xffffffffu, mbar_wait(bars.done(), 0, ctx)) != 0;
      tc_fence_after();
      const float inv = p.splits > 1 ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
      const int64_t part = ((static_cast<int64_t>(w.b) * p.a.max_q + qi) * p.a.Hq + hq) * p.splits + w.split;
      if (p.splits > 1 && mine) p.ml[part] = make_float2(m, l);
      T* dst = static_cast<T*>(p.o) + tok * p.a.o_token_stride + static_cast<int64_t>(hq) * p.a.o_head_stride;
#pragma unroll
      for (int c = 0; c < DP; c += 16) {
        if (c < D) {
          uint32_t v[16];
          tmem_ld16(o_mem + c, v);
          tmem_wait_ld();
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

template <typename T, int DP>
cudaError_t launch(const AttnArgs& p, unsigned grid, cudaStream_t stream) {
  static int attr_set[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(pq_kv8_tiles<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, attn_smem(DP));
    if (e != cudaSuccess) return e;
    if (dev < 64) attr_set[dev] = 1;
  }
  pq_kv8_tiles<T, DP><<<grid, kThreads, attn_smem(DP), stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

// From about 40 query rows of a cache head on: a block's step costs the same for 1 to
// 128 rows here, and in pq_kv8_rows it grows with every 16 (D = 128, rows of a head, here
// against there: one sequence of 4000, 24 rows 21 / 21 us, 48 22 / 25; 32 sequences of 3000, 32 rows
// 111 / 87, 48 111 / 123, 64 112 / 150).
bool attn_tc_takes(const pq_kv8_cache& c, const pq_kv8_attn& a) {
  return a.type != PQ_F32 && c.D <= 128 && static_cast<int64_t>(a.max_q) * (a.Hq / c.Hkv) > 40;
}

cudaError_t launch_attn_tc(const AttnArgs& p, unsigned grid, cudaStream_t stream) {
  if (p.a.type == PQ_F16) return p.c.D <= 64 ? launch<__half, 64>(p, grid, stream) : launch<__half, 128>(p, grid, stream);
  return p.c.D <= 64 ? launch<__nv_bfloat16, 64>(p, grid, stream) : launch<__nv_bfloat16, 128>(p, grid, stream);
}

}  // namespace pq
