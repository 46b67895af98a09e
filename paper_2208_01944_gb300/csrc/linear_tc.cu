// Dense layer on 8-bit codes for many tokens, on the 5th-generation tensor cores.
//
// Mathematics.  acc[m, n] = sum_k q[m, k] w[n, k], exact.  sm_103a has no 8-bit integer
// tcgen05 kind (and mma.sync on 8-bit integers runs at 158 TOPS), but 8-bit codes
// are exact half values: kind::f16 multiplies them exactly and its fp32 sums of
// integers stay exact below 2^24, that is for 1024 of K (127 * 128 * 1024 < 2^24).  Every
// 1024 of K the sums move from tensor memory into int32 registers; two accumulators
// take turns, so that one is read while the other is written.
//
// Tile.  128 output channels (the MMA's rows) x BN tokens (its columns) a block.  The
// weights stay 8-bit in memory: four warps turn each 128 x 64 block into halves and put
// it into tensor memory, from where the MMA takes its first operand, so the halves cost
// neither memory traffic nor shared-memory bandwidth.  The tokens come as halves
// (PQ_CODES_F16, written by the token quantiser) by TMA, in the 128-byte swizzle that
// the MMA reads.  With many tiles two blocks work as a pair (cta_group::2): 256 channels
// x BN tokens, each block holding half of the tokens, so that an SM takes in
// (8 + BN / 16) KB for each 64 of K instead of (8 + BN / 8).  Single blocks of 128 x 192 were bound by
// that: 32 KB in every 384 cycles is more than the 64 bytes a cycle that L2 gives an SM.
// Bound by the tensor rate for many tokens, by the weights' bytes for few.
//
// Roles (20 warps): 0 and 2 load (weights, tokens), 1 issues the MMAs (of the pair, in
// its first block), 4-7 and 8-11 convert a half each of every stage, 12-19 drain and
// write.  A stage is 128 of K: waiting for one and freeing it costs the issuing warp about
// 130 cycles beside its MMAs, more than there are to spare with stages of 64.  Few
// tiles: the blocks of a cluster take parts of K of one tile and add their int32 sums
// through distributed shared memory (in a fixed order; exact anyway).  Measured, the product alone: 8192 x 8192 x 8192
// 560 us (1.96 PFLOP/s), 2048 x 4096 x 4096 47 us, 48 x 8192 x 4096 14.5 us (2.3 TB/s of weights).
#include <cuda_runtime.h>

#include <algorithm>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_linear.h"
#include "pq_tc.cuh"
#include "pq_tokens.cuh"

namespace pq {
namespace {

constexpr int kTcThreads = 640;     // warpgroups: 0 loads and MMAs, 1 and 2 convert, 3 and 4 drain
constexpr int kTcBK = 128;          // K of one stage: 128 bytes of a weight row, twice 128 of a token row
constexpr int kTcExact = 8;         // stages whose fp32 sums are exact
constexpr int kTcWBytes = 128 * kTcBK;
constexpr int kTcMaxStages = 8;

// Tokens' rows of a block, the bytes of its stage, and the stages that fit.
__host__ __device__ constexpr int tc_rows(int BN, bool pair) { return pair ? BN / 2 : BN; }
__host__ __device__ constexpr int tc_stage_bytes(int BN, bool pair) { return kTcWBytes + tc_rows(BN, pair) * 256; }
__host__ __device__ constexpr int tc_stages(int BN, bool pair) {
  return 204800 / tc_stage_bytes(BN, pair) < kTcMaxStages ? 204800 / tc_stage_bytes(BN, pair) : kTcMaxStages;
}
__host__ __device__ constexpr int tc_smem(int BN, bool pair) {
  return tc_stages(BN, pair) * tc_stage_bytes(BN, pair) + 1024 /* alignment */ + 512 /* barriers */;
}
// Half stages of converted weights in tensor memory, 32 columns each, beside two accumulators.
__host__ __device__ constexpr int tc_a_slots(int BN) { return BN <= 128 ? 8 : BN <= 160 ? 6 : 4; }

// Barriers, 8 bytes each: loaded (a stage's bytes), full (its weights are halves too, in
// both blocks of a pair), empty (a ring each), a_empty (a slot of converted weights is
// free), acc_full, acc_empty (two each), done.
struct TcBars {
  uint32_t base;
  __device__ uint32_t loaded(int s) const { return base + 8u * s; }
  __device__ uint32_t full(int s) const { return base + 8u * (kTcMaxStages + s); }
  __device__ uint32_t empty(int s) const { return base + 8u * (2 * kTcMaxStages + s); }
  __device__ uint32_t a_empty(int s) const { return base + 8u * (3 * kTcMaxStages + s); }
  __device__ uint32_t acc_full(int i) const { return base + 8u * (4 * kTcMaxStages + i); }
  __device__ uint32_t acc_empty(int i) const { return base + 8u * (4 * kTcMaxStages + 2 + i); }
  __device__ uint32_t done() const { return base + 8u * (4 * kTcMaxStages + 4); }
};

// Instruction descriptor of kind::f16: half operands, fp32 sums, K-major.
__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N) {
  return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// Four MMAs (64 of K) with the first operand in tensor memory; the whole warp calls, one lane issues.
#define PQ_TC_MMA_X4(group)                                                                                            \
  asm volatile(                                                                                                        \
      "{\n.reg .pred p, q, e;\nelect.sync _|e, 0xffffffff;\nsetp.ne.b32 p, %10, 0;\nsetp.eq.b32 q, 0, 0;\n"            \
      "@e tcgen05.mma.cta_group::" group ".kind::f16 [%0], [%1], %5, %9, p;\n"                                         \
      "@e tcgen05.mma.cta_group::" group ".kind::f16 [%0], [%2], %6, %9, q;\n"                                         \
      "@e tcgen05.mma.cta_group::" group ".kind::f16 [%0], [%3], %7, %9, q;\n"                                         \
      "@e tcgen05.mma.cta_group::" group ".kind::f16 [%0], [%4], %8, %9, q;\n}" ::"r"(d),                              \
      "r"(a), "r"(a + 8), "r"(a + 16), "r"(a + 24), "l"(b), "l"(b + 2), "l"(b + 4), "l"(b + 6), "r"(idesc),            \
      "r"(accumulate)                                                                                                  \
      : "memory")
template <bool PAIR>
__device__ __forceinline__ void tc_mma_f16_ts_x4(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if (PAIR)
    PQ_TC_MMA_X4("2");
  else
    PQ_TC_MMA_X4("1");
}
#undef PQ_TC_MMA_X4

// Arrive once the MMAs issued so far are done: here, or on the same barrier of both blocks of the pair.
template <bool PAIR>
__device__ __forceinline__ void tc_commit_group(uint32_t bar) {
  if (PAIR)
    asm volatile(
        "{\n.reg .pred e;\nelect.sync _|e, 0xffffffff;\n"
        "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}" ::"r"(bar),
        "h"(static_cast<uint16_t>(3))
        : "memory");
  else
    tc_commit_warp(bar);
}

template <bool PAIR>
__device__ __forceinline__ void tmem_alloc_group(uint32_t dst_smem, uint32_t ncols) {
  if (PAIR) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(ncols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    tmem_alloc(dst_smem, ncols);
  }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_dealloc_group(uint32_t taddr, uint32_t ncols) {
  if (PAIR)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
  else
    tmem_dealloc(taddr, ncols);
}

__device__ __forceinline__ int4 load_of_peer(uint32_t addr, uint32_t rank) {
  uint32_t a;
  int4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(a)
               : "memory");
  return v;
}

// Arrive on a barrier of the pair's first block.  What it announces (tensor memory
// written or read) is ordered by the tcgen05 fences around it; a release at cluster
// scope would wait for this thread's stores to memory, and made a tile three times slower.
__device__ __forceinline__ void arrive_at_first(uint32_t bar) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(bar));
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(a) : "memory");
}

// One channel's results of kCols tokens from m on: the warp's 32 lanes write 32
// consecutive channels of one token at a time.  s_x: the tokens' scales in shared memory.
template <int kCols, typename T>
__device__ __forceinline__ void put_column_as(const LinearArgs& a, int64_t m, int n, const int32_t (&sum)[kCols],
                                              const float* s_x) {
  const float s_w = a.s_w[n], bias = a.bias != nullptr ? a.bias[n] : 0.0f;
  const bool add = a.bias != nullptr;
  const int left = static_cast<int>(min(static_cast<int64_t>(kCols), a.M - m));
  T* y = static_cast<T*>(a.y) + m * a.ldy + n;
  const float4* s4 = reinterpret_cast<const float4*>(s_x);
#pragma unroll
  for (int j = 0; j < kCols; j += 4) {
    const float4 f = s4[j / 4];
    float v[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = __fmul_rn(__fmul_rn(__int2float_rn(sum[j + i]), v[i]), s_w);
      if (add) v[i] = __fadd_rn(v[i], bias);
      if (j + i < left) *y = from_f32<T>(v[i]);
      y += a.ldy;
    }
  }
}

// Four channels of a token.
__device__ __forceinline__ void put_results4(const LinearArgs& a, int64_t m, int n, int4 acc, float s_x,
                                             const float (&s_w)[4], const float (&bias)[4], bool wide) {
  const int sums[4] = {acc.x, acc.y, acc.z, acc.w};
  if (!wide) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < a.N) put_result(a, m, n + i, sums[i], s_x, s_w[i], bias[i]);
    return;
  }
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = __fmul_rn(__fmul_rn(__int2float_rn(sums[i]), s_x), s_w[i]);
    if (a.bias != nullptr) y[i] = __fadd_rn(y[i], bias[i]);
  }
  const int64_t at = m * a.ldy + n;
  if (a.y_type == PQ_F32) {
    *reinterpret_cast<float4*>(static_cast<float*>(a.y) + at) = make_float4(y[0], y[1], y[2], y[3]);
    return;
  }
  uint2 h;
  if (a.y_type == PQ_F16) {
    h = make_uint2(pack_half2(y[0], y[1]), pack_half2(y[2], y[3]));
  } else {
    const __nv_bfloat162 b[2] = {__floats2bfloat162_rn(y[0], y[1]), __floats2bfloat162_rn(y[2], y[3])};
    memcpy(&h, b, sizeof(h));
  }
  *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.y) + at) = h;
}

template <int kCols>
__device__ __forceinline__ void put_column(const LinearArgs& a, int64_t m, int n, const int32_t (&sum)[kCols],
                                           const float* s_x) {
  if (n >= a.N) return;
  if (a.acc != nullptr) {
#pragma unroll
    for (int j = 0; j < kCols; ++j)
      if (m + j < a.M) a.acc[(m + j) * a.N + n] = sum[j];
  }
  if (a.y == nullptr) return;
  if (a.y_type == PQ_F32)
    put_column_as<kCols, float>(a, m, n, sum, s_x);
  else if (a.y_type == PQ_F16)
    put_column_as<kCols, __half>(a, m, n, sum, s_x);
  else
    put_column_as<kCols, __nv_bfloat16>(a, m, n, sum, s_x);
}

// Tokens j, j + 8, .. of a tile below `end`, U of them: four channels of each, summed over the cluster's
// parts, I at a time, and written.  U x I loads from the peers are on their way together (one after the
// other, a call of 48 x 8192 x 4096 spent 2.4 of its 16.3 us here, now 1.4 of 15.3).
template <int U, int I, int kCols>
__device__ __forceinline__ void add_parts(const LinearTc& p, uint32_t from, int j, int end, const float (&scales)[8][kCols],
                                          int64_t m0, int n, const float (&s_w)[4], const float (&bias)[4], bool wide) {
  int4 sums[U] = {};
  for (int b = 0; b < p.k_parts; b += I) {
    int4 v[I][U] = {};
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (b + i < p.k_parts && j + 8 * u < end) v[i][u] = load_of_peer(from + (j + 8 * u) * 512, b + i);
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int u = 0; u < U; ++u)
        sums[u].x += v[i][u].x, sums[u].y += v[i][u].y, sums[u].z += v[i][u].z, sums[u].w += v[i][u].w;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int t = j + 8 * u;
    if (t < end) put_results4(p.a, m0 + t, n, sums[u], scales[4 * (t / kCols)][t % kCols], s_w, bias, wide);
  }
}

// Tile t: channel tiles in bands, the tokens' tiles along a band, so that the tiles
// at work at one time share weights and tokens in L2.
__device__ __forceinline__ void tile_origin(const LinearTc& p, int t, int channels, int BN, int* n0, int64_t* m0) {
  const int high = 2048 / channels;  // channel tiles of a band
  const int band = t / (high * p.m_tiles), in = t - band * high * p.m_tiles;
  const int width = min(high, p.n_tiles - band * high);
  *n0 = (band * high + in % width) * channels;
  *m0 = static_cast<int64_t>(in / width) * BN;
}

template <int BN, bool PAIR>
__global__ void __launch_bounds__(kTcThreads, 1)
    pq_linear_tc(const __grid_constant__ LinearTc p, const __grid_constant__ CUtensorMap map_w,
                 const __grid_constant__ CUtensorMap map_q) {
  constexpr int kStages = tc_stages(BN, PAIR);
  constexpr int kSlots = tc_a_slots(BN);
  constexpr int kTok = tc_rows(BN, PAIR) * 128;  // bytes of 64 of K of the block's tokens
  constexpr int kCols = BN / 2;           // columns of an accumulator that one of its two draining warps takes
  constexpr int kStep = kCols % 32 == 0 ? 32 : 16;
  constexpr uint32_t kABase = 2 * BN;     // first tensor-memory column of the weights' stages
  constexpr int kChannels = PAIR ? 256 : 128;
  static_assert(kABase + 32 * kSlots <= 512 && kSlots <= kTcMaxStages && kStages >= 3, "memory");
  extern __shared__ uint8_t raw[];
  __shared__ int abort_flag;
  __shared__ uint32_t tmem_base;
  __shared__ alignas(16) float scales[8][kCols];  // of each draining warp's tokens
  const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t tok_base = smem, w_base = smem + kStages * 2 * kTok;
  const TcBars bars{w_base + kStages * kTcWBytes};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = PAIR || p.k_parts > 1 ? static_cast<int>(cluster_rank()) : 0;

  if (warp == 2 && lane == 0) {
    prefetch_tmap(&map_w);
    prefetch_tmap(&map_q);
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(bars.loaded(s), 2);
      mbar_init(bars.full(s), PAIR ? 16 : 8);
      mbar_init(bars.empty(s), 1);
    }
    for (int s = 0; s < kSlots; ++s) mbar_init(bars.a_empty(s), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bars.acc_full(i), 1);
      mbar_init(bars.acc_empty(i), PAIR ? 16 : 8);
    }
    mbar_init(bars.done(), 1);
    abort_flag = 0;
    fence_mbar_init();
  }
  if (PAIR) cluster_sync();  // the other block arrives on these barriers
  if (warp == 1) tmem_alloc_group<PAIR>(smem_u32(&tmem_base), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;

  // this block's part of K, in stages, and its tiles
  const int all = (p.a.K + kTcBK - 1) / kTcBK;
  const int kb0 = PAIR ? 0 : static_cast<int>(static_cast<int64_t>(all) * rank / p.k_parts);
  const int kbs = PAIR ? all : static_cast<int>(static_cast<int64_t>(all) * (rank + 1) / p.k_parts) - kb0;
  const int share = PAIR ? 2 : p.k_parts;  // blocks of one tile
  const int first_tile = blockIdx.x / share, tile_step = gridDim.x / share;
  const int tiles = p.n_tiles * p.m_tiles;
  WaitCtx ctx{&abort_flag, p.err, p.wait_limit_ns, PQ_ERR_PRODUCER};

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if ((warp == 0 || warp == 2) && lane == 0) {
      // ---- loads: the weights (warp 0), which do not depend on the kernel before this
      // one, and the tokens.  One thread for both took longer for a stage than its MMAs do.
      const bool weights = warp == 0;
      Ring r;
      bool ok = true;
      int issued = 0;
      if (!weights) wait_previous_kernel();
      for (int t = first_tile; ok && t < tiles; t += tile_step) {
        int n0;
        int64_t m0;
        tile_origin(p, t, kChannels, BN, &n0, &m0);
        const int row = weights ? n0 + (PAIR ? 128 * rank : 0) : static_cast<int>(m0) + (PAIR ? BN / 2 * rank : 0);
        for (int kb = 0; kb < kbs; ++kb, ++issued) {
          if (issued >= kStages && !mbar_wait(bars.empty(r.s), r.phase ^ 1u, ctx)) {
            ok = false;
            break;
          }
          const uint32_t bar = bars.loaded(r.s);
          const int k = (kb0 + kb) * kTcBK;
          mbar_arrive_expect_tx(bar, weights ? kTcWBytes : 2 * kTok);
          if (weights) {
            tma_load_2d(w_base + r.s * kTcWBytes, &map_w, k, row, bar);
          } else {
            tma_load_2d(tok_base + r.s * 2 * kTok, &map_q, k, row, bar);
            tma_load_2d(tok_base + r.s * 2 * kTok + kTok, &map_q, k + 64, row, bar);
          }
          r.next(kStages);
        }
      }
      // What was loaded last may still be on its way.  After a wait that ran out, one of
      // the two may have stopped short of the other, whose last stages then never fill:
      // their own wait ends at its limit.
      for (int k = max(0, issued - kStages); k < issued; ++k)
        mbar_wait_drain(bars.loaded(k % kStages), (k / kStages) & 1, p.wait_limit_ns, p.err);
    } else if (warp == 1 && (!PAIR || rank == 0)) {
      // ---- MMAs
      ctx.err_bits = PQ_ERR_MMA;
      constexpr uint32_t idesc = idesc_f16_f32(kChannels, BN);
      auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, ctx)) != 0; };
      Ring r;
      int slot = 0;
      uint32_t stretch = 0;  // exact stretches of K so far, over all tiles
      bool ok = true;
      for (int t = first_tile; ok && t < tiles; t += tile_step) {
        for (int c0 = 0; ok && c0 < kbs; c0 += kTcExact, ++stretch) {
          const int c1 = min(kbs, c0 + kTcExact);
          const uint32_t acc = stretch & 1, uses = stretch >> 1;
          if (uses > 0) ok = wait(bars.acc_empty(acc), (uses - 1) & 1);
          for (int kb = c0; ok && kb < c1; ++kb) {
            ok = wait(bars.full(r.s), r.phase);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              tc_mma_f16_ts_x4<PAIR>(tmem + acc * BN, tmem + kABase + 32 * slot,
                                     sw128_desc(tok_base + (2 * r.s + h) * kTok), idesc, h > 0 || kb != c0);
              tc_commit_group<PAIR>(bars.a_empty(slot));
              if (++slot == kSlots) slot = 0;
            }
            tc_commit_group<PAIR>(bars.empty(r.s));
            r.next(kStages);
          }
          if (ok) tc_commit_group<PAIR>(bars.acc_full(acc));
        }
      }
      // every MMA issued must be over before the tensor memory is given back
      tc_commit_group<PAIR>(bars.done());
      if (lane == 0) mbar_wait_drain(bars.done(), 0, p.wait_limit_ns, p.err);
      __syncwarp();
    }
  } else if (warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    // ---- weights to halves: this thread's row of every block, one half (64 of K) of it
    ctx.err_bits = PQ_ERR_EPILOGUE;
    const int row = 32 * (warp & 3) + lane, half = (warp - 4) >> 2;
    const uint32_t swizzle = row & 7;
    const uint32_t to = tmem + kABase + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
    const int total = first_tile < tiles ? ((tiles - first_tile - 1) / tile_step + 1) * kbs : 0;
    Ring r;
    int slot = half;
    uint32_t round = 0;  // times that the slot was used before
    for (int i = 0; i < total; ++i) {
      if (!__all_sync(0xffffffffu, mbar_wait(bars.loaded(r.s), r.phase, ctx))) break;
      const uint32_t src = w_base + r.s * kTcWBytes + row * kTcBK;
      uint32_t h[32];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint4 v = lds128(src + (((4 * half + c) ^ swizzle) << 4));
        half_of_codes(v.x, h[8 * c], h[8 * c + 1]);
        half_of_codes(v.y, h[8 * c + 2], h[8 * c + 3]);
        half_of_codes(v.z, h[8 * c + 4], h[8 * c + 5]);
        half_of_codes(v.w, h[8 * c + 6], h[8 * c + 7]);
      }
      if (round > 0 && !__all_sync(0xffffffffu, mbar_wait(bars.a_empty(slot), (round - 1) & 1, ctx))) break;
      tc_fence_after();
      tmem_st32(to + 32 * slot, h);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR)
          arrive_at_first(bars.full(r.s));
        else
          mbar_arrive(bars.full(r.s));
      }
      r.next(kStages);
      slot += 2;
      if (slot >= kSlots) slot = half, ++round;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 144;");
    // ---- sums and outputs: this thread's channel, half of each accumulator's tokens
    ctx.err_bits = PQ_ERR_EPILOGUE;
    const int quarter = warp & 3, side = (warp - 12) >> 2;
    const uint32_t from = tmem + (static_cast<uint32_t>(32 * quarter) << 16) + side * kCols;
    wait_previous_kernel();  // the tokens' scales
    int32_t sum[kCols];
    uint32_t stretch = 0;
    bool ok = true;
    for (int t = first_tile; ok && t < tiles; t += tile_step) {
      int n0;
      int64_t m0;
      tile_origin(p, t, kChannels, BN, &n0, &m0);
      __syncwarp();
      for (int j = lane; j < kCols; j += 32) {
        const int64_t m = m0 + side * kCols + j;
        scales[warp - 12][j] = p.a.s_x != nullptr && m < p.a.M ? p.a.s_x[m] : 0.0f;
      }
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kCols; ++j) sum[j] = 0;
      for (int c0 = 0; ok && c0 < kbs; c0 += kTcExact, ++stretch) {
        const uint32_t acc = stretch & 1;
        ok = __all_sync(0xffffffffu, mbar_wait(bars.acc_full(acc), (stretch >> 1) & 1, ctx)) != 0;
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int j = 0; j < kCols; j += kStep) {
          uint32_t v[kStep];
          if constexpr (kStep == 32)
            tmem_ld32(from + acc * BN + j, v);
          else
            tmem_ld16(from + acc * BN + j, v);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < kStep; ++i) sum[j + i] += __float2int_rn(__uint_as_float(v[i]));
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR)
            arrive_at_first(bars.acc_empty(acc));
          else
            mbar_arrive(bars.acc_empty(acc));
        }
      }
      if (!ok) break;
      if (!PAIR && p.k_parts > 1) {
        // the ring is idle: this block's only tile is over (the last accumulator was full)
#pragma unroll
        for (int j = 0; j < kCols; ++j)
          asm volatile("st.shared.s32 [%0], %1;" ::"r"(tok_base + ((side * kCols + j) * 128 + 32 * quarter + lane) * 4),
                       "r"(sum[j])
                       : "memory");
        break;
      }
      put_column<kCols>(p.a, m0 + side * kCols, n0 + (PAIR ? 128 * rank : 0) + 32 * quarter + lane, sum, scales[warp - 12]);
    }
    if (!PAIR && p.k_parts > 1) {
      // add the cluster's parts: every block writes a share of the tokens, a warp one
      // token's 128 channels at a time, four a lane, whose scales it has by then
      int n0;
      int64_t m0;
      tile_origin(p, first_tile, kChannels, BN, &n0, &m0);
      const int n = n0 + 4 * lane;
      float s_w[4], bias[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s_w[i] = p.a.s_w != nullptr && n + i < p.a.N ? p.a.s_w[n + i] : 0.0f;
        bias[i] = p.a.bias != nullptr && n + i < p.a.N ? p.a.bias[n + i] : 0.0f;
      }
      // four channels of a token in one store
      const bool wide = n + 4 <= p.a.N && p.a.acc == nullptr && p.a.ldy % 4 == 0 &&
                        reinterpret_cast<uintptr_t>(p.a.y) % (p.a.y_type == PQ_F32 ? 16 : 8) == 0;
      cluster_sync();
      const int j1 = static_cast<int>(min(static_cast<int64_t>(BN * (rank + 1) / p.k_parts), p.a.M - m0));
      const int j0 = BN * rank / p.k_parts + warp - 12;
      if (ok && j0 + 8 >= j1) {
        if (j0 < j1) add_parts<1, 8>(p, tok_base + 16 * lane, j0, j1, scales, m0, n, s_w, bias, wide);
      } else if (ok) {
        for (int j = j0; j < j1; j += 32) add_parts<4, 2>(p, tok_base + 16 * lane, j, j1, scales, m0, n, s_w, bias, wide);
      }
      cluster_sync();
    }
  }
  // the blocks of a cluster leave together: their sums are read by the others
  if (!PAIR && p.k_parts > 1 && warp < 12) {
    cluster_sync();
    cluster_sync();
  }
  tc_fence_before();
  __syncthreads();
  // a pair's MMAs work on both blocks' memory, and its barriers are arrived on from both
  if (PAIR) cluster_sync();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc_group<PAIR>(tmem, 512);
  }
}

template <int BN, bool PAIR>
cudaError_t launch(const LinearTc& p, const CUtensorMap& w, const CUtensorMap& q, int sms, bool after_tokens,
                   cudaStream_t stream) {
  static int most[64] = {0};  // clusters of two that fit the device at one time
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64) return cudaErrorInvalidDevice;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kTcThreads);
  cfg.dynamicSmemBytes = tc_smem(BN, PAIR);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  const int cluster = PAIR ? 2 : p.k_parts;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(cluster);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  if (most[dev] == 0) {
    e = cudaFuncSetAttribute(pq_linear_tc<BN, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, tc_smem(BN, PAIR));
    if (e != cudaSuccess) return e;
    int n = sms;
    if (PAIR) {
      cfg.gridDim = dim3(static_cast<unsigned>(sms / 2 * 2));
      cfg.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&n, pq_linear_tc<BN, PAIR>, &cfg);
      if (e != cudaSuccess || n < 1) return e != cudaSuccess ? e : cudaErrorInvalidConfiguration;
    }
    most[dev] = n;
  }
  const int64_t tiles = static_cast<int64_t>(p.n_tiles) * p.m_tiles;
  // a cluster that shares K has one tile; otherwise as many blocks as there are at one time take the tiles in turn
  const int64_t at_once = p.k_parts > 1 ? tiles : std::min<int64_t>(tiles, most[dev]);
  cfg.gridDim = dim3(static_cast<unsigned>(at_once * cluster));
  cfg.numAttrs = after_tokens ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, pq_linear_tc<BN, PAIR>, p, w, q);
}

}  // namespace

bool linear_tc_takes(const LinearArgs& a) {
  return is_aligned(a.q, 16) && a.ldq % 8 == 0 && is_aligned(a.w, 16) && a.ldw % 16 == 0 && a.M <= (1ll << 30);
}

cudaError_t launch_linear_tc(const LinearArgs& a, bool after_tokens, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  LinearTc p = {};
  p.a = a;
  p.err = device_error_word();
  p.wait_limit_ns = wait_limit_ns();
  if (p.err == nullptr) return cudaErrorInitializationError;
  // Tiles.  Up to 128 tokens: single blocks, one tile of tokens, the fewest columns
  // that hold them.  More: the cheaper of single blocks of 128 tokens and pairs of 160
  // or 192, by rounds of tiles x the time of 64 of K, which was 404 and 423 cycles for
  // the pairs and 384 for pairs of 128 (about bn + 500 in units of 0.6 cycles), which never take
  // fewer rounds than single blocks of 128.  Single blocks share K while the
  // chip is less than half full and each part keeps 256 of K; eight parts of 128 tokens
  // take longer to add than they save (16 tiles of K = 8192: 22 us, four parts 15 us), and
  // of clusters of eight only one or two fit a part of the chip at a time (64 tokens, K = 8192: 16
  // tiles 20.6 us, in four parts 14.7; 8 tiles 10.7, in four parts 13.4).
  auto ceil_div = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
  int bn = a.M <= 32 ? 32 : a.M <= 64 ? 64 : 128;
  const int64_t singles = ceil_div(a.N, 128) * ceil_div(a.M, bn);
  p.k_parts = 1;
  for (int c = 2; c <= (bn < 128 ? 8 : 4) && singles * c <= (c == 8 ? sms / 2 : sms) && a.K / c >= 256; c *= 2) p.k_parts = c;
  bool pair = false;
  if (a.M > 128) {
    double best = static_cast<double>(ceil_div(singles * p.k_parts, sms)) * (bn + 500) / p.k_parts;
    for (int c = 192; c >= 160; c -= 32) {
      const double cost =
          static_cast<double>(ceil_div(ceil_div(a.N, 256) * ceil_div(a.M, c), std::max(1, sms / 2))) * (c + 500);
      if (cost < best) best = cost, bn = c, pair = true;
    }
  }
  if (pair) p.k_parts = 1;
  p.n_tiles = static_cast<int>(ceil_div(a.N, pair ? 256 : 128));
  const int64_t m_tiles = ceil_div(a.M, bn);
  if (p.n_tiles * m_tiles > 0x7FFFFFFF) return cudaErrorInvalidValue;
  p.m_tiles = static_cast<int>(m_tiles);
  CUtensorMap w, q;
  if (!encode_map_2d(&w, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.w, static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.N),
                     static_cast<uint64_t>(a.ldw), kTcBK, 128, CU_TENSOR_MAP_SWIZZLE_128B) ||
      !encode_map_2d(&q, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, a.q, static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.M),
                     static_cast<uint64_t>(a.ldq) * 2, 64, static_cast<uint32_t>(pair ? bn / 2 : bn),
                     CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorInvalidValue;
  if (pair && bn == 192) return launch<192, true>(p, w, q, sms, after_tokens, stream);
  if (pair) return launch<160, true>(p, w, q, sms, after_tokens, stream);
  if (bn == 32) return launch<32, false>(p, w, q, sms, after_tokens, stream);
  if (bn == 64) return launch<64, false>(p, w, q, sms, after_tokens, stream);
  return launch<128, false>(p, w, q, sms, after_tokens, stream);
}

}  // namespace pq
