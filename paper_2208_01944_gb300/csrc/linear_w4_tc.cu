// Dense layers with 4-bit weights for a batch of tokens, on the 5th-generation tensor cores.
//
// Mathematics.  For each group of input channels, kind::f16 multiplies the codes (integers, exact in the activations' type) with
// the activations into an accumulator of its own, in fp32; it is read back, multiplied with the channel's scale of the group and
// added in registers, in fp32.  So a weight is never rounded: scaled to 16 bits before the product it would be, by as much as the
// output is.
//
// Tile.  128 output channels (8 packed strips) x BN tokens a block.  Codes stay 4-bit in memory and shared memory; sixteen warps turn
// them into 16-bit operands in tensor memory, which take no shared-memory bandwidth: a lane's packed 16 bytes are, unpacked, the
// registers of a 16 x 256-bit store, so nothing is exchanged between lanes.  Activations come by TMA in the 128-byte swizzle.
// The accumulators of groups take turns, so that one is read while others are written.  Few tiles: the blocks of a cluster take
// parts of K of one tile and add their fp32 sums through distributed shared memory, in order.
//
// Bound by hand-overs between the roles where tokens are few (no pipe above 40 %), by reading groups' accumulators where they are many.
// Measured, bf16: 48 x 8192 x 4096 with groups of 64 17 us (1.1 TB/s of weights), 2048 x 4096 x 4096 with groups of 128 86 us (0.80
// PFLOP/s), of 64 111, of 32 183.
//
// Roles (32 warps): 0 and 2 load (weights, tokens), 4-19 unpack, 20-27 drain and write, 28-31 issue the MMAs.  A stage is 128 of K.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_linear.h"
#include "pq_tc.cuh"
#include "pq_tokens.cuh"
#include "pq_w4.cuh"
#include "pq_w4_turns.h"

namespace pq {
namespace {

constexpr int kThreads = 1024;
constexpr int kJoin = 8;  // tokens that a thread adds up at one time
using w4::job_k;
using w4::kAColumns;
using w4::kMaxSlots;
using w4::kMaxStages;
using w4::kWBytes;
using w4::places;
using w4::slots;
using w4::smem_bytes;
using w4::stages;
static_assert(w4::kBlockK == kBlockK && kWBytes == kTileStrips * (1024 + 256), "a stage");

struct W4Tc {
  W4Args a;
  int n_tiles, m_tiles;  // tiles of 128 channels, of BN tokens
  int k_parts;           // blocks of a cluster that share a tile's K (1: none)
  unsigned int* err;
  uint64_t wait_limit_ns;
};

// Barriers: loaded (a stage's bytes), full (a slot is unpacked), acc_full (a place's MMAs are over); stage_empty, slot_empty and
// acc_empty (the job's sums are read, and with them everything that they came from), done.  A wait or a commit takes a warp
// among these 32 some 50 to 200 cycles, more than an MMA of these tiles: so one commit a job, and the draining warps free all.
struct Bars {
  uint32_t base;
  __device__ uint32_t loaded(int s) const { return base + 8u * s; }
  __device__ uint32_t stage_empty(int s) const { return base + 8u * (kMaxStages + s); }
  __device__ uint32_t full(int s) const { return base + 8u * (2 * kMaxStages + s); }
  __device__ uint32_t slot_empty(int s) const { return base + 8u * (2 * kMaxStages + kMaxSlots + s); }
  __device__ uint32_t acc_full(int s) const { return base + 8u * (2 * kMaxStages + 2 * kMaxSlots + s); }
  __device__ uint32_t acc_empty(int s) const { return base + 8u * (2 * kMaxStages + 3 * kMaxSlots + s); }
  __device__ uint32_t done() const { return base + 8u * (2 * kMaxStages + 4 * kMaxSlots); }
};
constexpr int kBars = 2 * kMaxStages + 4 * kMaxSlots + 1;

// Instruction descriptor of kind::f16: halves or bfloat16, fp32 sums, K-major.
template <typename T>
__host__ __device__ constexpr uint32_t idesc_of(int N) {
  return (1u << 4) | (std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u) | (static_cast<uint32_t>(N >> 3) << 17) |
         (static_cast<uint32_t>(128 >> 4) << 24);
}

// Two MMAs (32 of K) with the first operand in tensor memory; the whole warp calls, one lane issues.
__device__ __forceinline__ void mma_ts_x2(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p, q, e;\nelect.sync _|e, 0xffffffff;\nsetp.ne.b32 p, %6, 0;\nsetp.eq.b32 q, 0, 0;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %3, %5, p;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%2], %4, %5, q;\n}" ::"r"(d),
      "r"(a), "r"(a + 8), "l"(b), "l"(b + 2), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Four MMAs (64 of K).
__device__ __forceinline__ void mma_ts_x4(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p, q, e;\nelect.sync _|e, 0xffffffff;\nsetp.ne.b32 p, %10, 0;\nsetp.eq.b32 q, 0, 0;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %5, %9, p;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%2], %6, %9, q;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%3], %7, %9, q;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%4], %8, %9, q;\n}" ::"r"(d),
      "r"(a), "r"(a + 8), "r"(a + 16), "r"(a + 24), "l"(b), "l"(b + 2), "l"(b + 4), "l"(b + 6), "r"(idesc), "r"(accumulate)
      : "memory");
}

// 16 lanes x 32 columns: lane 4 g + t holds of lanes g and g + 8, for each 8 columns, columns 2 t and 2 t + 1.
__device__ __forceinline__ void tmem_st_16x256b_x4(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// (s0, s1) += m (a, b), packed.
__device__ __forceinline__ void fma_pair(float& s0, float& s1, float a, float b, float m) {
  asm("{\n.reg .b64 s, t, u;\nmov.b64 s, {%0, %1};\nmov.b64 t, {%2, %3};\nmov.b64 u, {%4, %4};\nfma.rn.f32x2 s, t, u, s;\nmov.b64 {%0, %1}, s;\n}"
      : "+f"(s0), "+f"(s1)
      : "f"(a), "f"(b), "f"(m));
}

__device__ __forceinline__ float load_of_peer_f32(uint32_t addr, uint32_t rank) {
  uint32_t a;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

__device__ __forceinline__ float scale_in_smem(uint32_t at, int type) {
  if (type == PQ_F32) {
    float f;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f) : "r"(at) : "memory");
    return f;
  }
  uint16_t h;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at) : "memory");
  return type == PQ_F16 ? __half2float(__ushort_as_half(h)) : __uint_as_float(static_cast<uint32_t>(h) << 16);
}

// Tile t: channel tiles in bands of 16, the tokens' tiles along a band, so that the tiles at work at one time share weights and tokens in L2.
__device__ __forceinline__ void tile_origin(const W4Tc& p, int t, int BN, int* n_tile, int64_t* m0) {
  const int band = t / (16 * p.m_tiles), in = t - band * 16 * p.m_tiles;
  const int width = min(16, p.n_tiles - band * 16);
  *n_tile = band * 16 + in % width;
  *m0 = static_cast<int64_t>(in / width) * BN;
}

// GS: log2(group).  PARTS: matrices of tokens, one below the other in map_x, whose products are added (three for fp32).
template <typename T, int BN, int GS, int PARTS>
__global__ void __launch_bounds__(kThreads, 1) pq_linear_w4_tc(const __grid_constant__ W4Tc p, const __grid_constant__ CUtensorMap map_x) {
  constexpr int kStages = stages(BN, PARTS);
  constexpr int kSlots = slots(GS), kPlaces = places(BN, GS);
  constexpr int kSlotColumns = kAColumns / kSlots;
  constexpr int kAccs = job_k(GS) >> GS;           // accumulators of a job
  constexpr int kPerStage = kBlockK / job_k(GS);   // jobs of a stage
  constexpr int kIssuers = w4::issuers(BN, GS);    // warps that issue jobs in turn
  constexpr int kTurns = w4::unpacking_sets(GS);   // sets of warps that unpack jobs in turn
  constexpr int kUnpackers = 16 / kTurns;          // warps of a set: 32 channels of 64 of K each
  static_assert(kSlots % kTurns == 0 && kSlots % kIssuers == 0 && kPlaces % kIssuers == 0 && kPlaces % 2 == 0 && kStages % 2 == 0, "turns");
  constexpr int kTok = BN * 128;   // bytes of 64 of K of the tokens
  // Two sides of draining warps: up to 64 tokens they take jobs in turn, each all of their columns (one side's way through a
  // job, 550 cycles, was the longest of all roles'); 128 tokens' sums do not fit a thread, there each takes half of the columns.
  constexpr bool kSplit = BN == 128;
  constexpr int kCols = kSplit ? BN / 2 : BN;
  constexpr int kDrainers = kSplit ? 8 : 4;        // warps that drain a job
  extern __shared__ uint8_t raw[];
  __shared__ alignas(8) uint64_t bar_words[kBars];
  __shared__ int abort_flag;
  __shared__ uint32_t tmem_base;
  const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t tok_base = smem, w_base = smem + kStages * PARTS * 2 * kTok;
  const Bars bars{smem_u32(bar_words)};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = p.k_parts > 1 ? static_cast<int>(cluster_rank()) : 0;
  const PackedW4& w = p.a.p;

  if (warp == 2 && lane == 0) prefetch_tmap(&map_x);
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(bars.loaded(s), 2);
      mbar_init(bars.stage_empty(s), kDrainers * kPerStage);
    }
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(bars.full(s), kUnpackers);
      mbar_init(bars.slot_empty(s), kDrainers);
    }
    for (int s = 0; s < kPlaces; ++s) {
      mbar_init(bars.acc_full(s), 1);
      mbar_init(bars.acc_empty(s), kDrainers);
    }
    mbar_init(bars.done(), kIssuers);
    abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc(smem_u32(&tmem_base), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // all 512 columns are this block's: the base is 0 (a constant address costs the issuing warps no register moves)
  constexpr uint32_t tmem = 0;

  // this block's part of K, in stages, and its tiles
  const int kb0 = static_cast<int>(static_cast<int64_t>(w.blocks) * rank / p.k_parts);
  const int kbs = static_cast<int>(static_cast<int64_t>(w.blocks) * (rank + 1) / p.k_parts) - kb0;
  const int first_tile = blockIdx.x / p.k_parts, tile_step = gridDim.x / p.k_parts;
  const int tiles = p.n_tiles * p.m_tiles;
  const int total = first_tile < tiles ? ((tiles - first_tile - 1) / tile_step + 1) * kbs * kPerStage : 0;  // jobs
  WaitCtx ctx{&abort_flag, p.err, p.wait_limit_ns, PQ_ERR_PRODUCER};

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if ((warp == 0 || warp == 2) && lane == 0) {
      // ---- loads: a stage's strips (warp 0), its tokens (warp 2)
      const bool weights = warp == 0;
      Ring r;
      bool ok = true;
      int issued = 0;
      if (!weights) wait_previous_kernel();  // it may have written the tokens' copy
      for (int t = first_tile; ok && t < tiles; t += tile_step) {
        int n_tile;
        int64_t m0;
        tile_origin(p, t, BN, &n_tile, &m0);
        const uint32_t bytes = w.pitch(n_tile * kTileStrips);
        const uint8_t* from = p.a.w + w.strip_at(n_tile * kTileStrips) + static_cast<int64_t>(kb0) * bytes;
        for (int kb = 0; kb < kbs; ++kb, ++issued) {
          if (issued >= kStages && !mbar_wait(bars.stage_empty(r.s), r.phase ^ 1u, ctx)) {
            ok = false;
            break;
          }
          const uint32_t bar = bars.loaded(r.s);
          if (weights) {
            mbar_arrive_expect_tx(bar, bytes);
            bulk_load(w_base + r.s * kWBytes, from, bytes, bar);
            from += bytes;
          } else {
            const int k = (kb0 + kb) * kBlockK;
            mbar_arrive_expect_tx(bar, PARTS * 2 * kTok);
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
              const uint32_t to = tok_base + (r.s * PARTS + part) * 2 * kTok;
              const int row = static_cast<int>(part * p.a.M + m0);  // (rows past the part's end are the next one's: not stored)
              tma_load_2d(to, &map_x, k, row, bar);
              tma_load_2d(to + kTok, &map_x, k + 64, row, bar);
            }
          }
          r.next(kStages);
        }
      }
      // what was loaded last may still be on its way
      for (int k = max(0, issued - kStages); k < issued; ++k)
        mbar_wait_drain(bars.loaded(k % kStages), (k / kStages) & 1, p.wait_limit_ns, p.err);
    }
  } else if (warp >= 28) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    // ---- MMAs: these warps issue jobs in turn (one warp alone, its scheduler shared with unpacking warps, took 1200 cycles for 128 of K)
    ctx.err_bits = PQ_ERR_MMA;
    if (warp - 28 < kIssuers) {
      constexpr uint32_t idesc = idesc_of<T>(BN);
      const int turn = warp - 28;
      // stage of job i: i / kPerStage modulo kStages
      int stage = turn / kPerStage;
      const int stage_step = kIssuers / kPerStage > 0 ? kIssuers / kPerStage : 1;
      uint32_t slot = turn, slot_phase = 0, place = turn, place_phase = 1;
      for (int i = turn; i < total; i += kIssuers) {
        if (!__all_sync(0xffffffffu, mbar_wait(bars.full(slot), slot_phase, ctx))) break;
        if (i >= kPlaces && !__all_sync(0xffffffffu, mbar_wait(bars.acc_empty(place), place_phase, ctx))) break;
        tc_fence_after();
        const uint32_t acc = tmem + kAColumns + place * (kAccs * BN), codes = tmem + slot * kSlotColumns;
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          const uint64_t tokens = sw128_desc(tok_base + ((stage * PARTS + part) * 2 + (kPerStage == 2 ? i & 1 : 0)) * kTok);
          if (GS == 7) {
            mma_ts_x4(acc, codes, tokens, idesc, part > 0);
            mma_ts_x4(acc, codes + 32, tokens + (kTok >> 4), idesc, 1);
          } else if (GS == 6) {
            mma_ts_x4(acc, codes, tokens, idesc, part > 0);
          } else {
            mma_ts_x2(acc, codes, tokens, idesc, part > 0);
            mma_ts_x2(acc + BN, codes + 16, tokens + 4, idesc, part > 0);
          }
        }
        tc_commit_warp(bars.acc_full(place));
        slot += kIssuers;
        if (slot >= kSlots) slot -= kSlots, slot_phase ^= 1u;
        place += kIssuers;
        if (place >= kPlaces) place -= kPlaces, place_phase ^= 1u;
        stage += stage_step;
        if (stage >= kStages) stage -= kStages;
      }
      // every MMA issued must be over before the tensor memory is given back
      tc_commit_warp(bars.done());
      if (lane == 0) mbar_wait_drain(bars.done(), 0, p.wait_limit_ns, p.err);
      __syncwarp();
    }
  } else if (warp < 20) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    // ---- codes to operands
    ctx.err_bits = PQ_ERR_EPILOGUE;
    const int quarter = warp & 3, set = (warp - 4) >> 2;
    const int turn = kPerStage == 1 ? set >> 1 : set, half = set & 1;  // (job i of 64 of K is half i % 2 of its stage)
    const uint32_t to = tmem + (kPerStage == 1 ? 32 * half : 0) + (static_cast<uint32_t>(32 * quarter) << 16);
    const uint32_t src = w_base + 2 * quarter * w.block_bytes + half * 512 + lane * 16;
    Ring r, slot;
    for (int i = 0; i < turn; ++i) slot.next(kSlots);
    for (int i = 0; i < turn / kPerStage; ++i) r.next(kStages);
    for (int i = turn; i < total; i += kTurns) {
      if (!__all_sync(0xffffffffu, mbar_wait(bars.loaded(r.s), r.phase, ctx))) break;
      uint32_t h[2][16];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint4 v = lds128(src + r.s * kWBytes + j * w.block_bytes);
        const uint32_t words[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t low[4], high[4];  // rows g and g + 8, 32 of K
          code_pairs<T>(words[2 * c], low);
          code_pairs<T>(words[2 * c + 1], high);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            h[j][8 * c + 4 * k] = low[2 * k], h[j][8 * c + 4 * k + 1] = low[2 * k + 1];
            h[j][8 * c + 4 * k + 2] = high[2 * k], h[j][8 * c + 4 * k + 3] = high[2 * k + 1];
          }
        }
      }
      if (i >= kSlots && !__all_sync(0xffffffffu, mbar_wait(bars.slot_empty(slot.s), slot.phase ^ 1u, ctx))) break;
      tc_fence_after();
#pragma unroll
      for (int j = 0; j < 2; ++j) tmem_st_16x256b_x4(to + slot.s * kSlotColumns + (static_cast<uint32_t>(16 * j) << 16), h[j]);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bars.full(slot.s));
      r.next(kStages);
      r.next(kStages);
      slot.s += kTurns;
      if (slot.s >= kSlots) slot.s -= kSlots, slot.phase ^= 1u;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    // ---- sums and outputs: this thread's channel; tiles of 128 tokens: half of each accumulator's
    ctx.err_bits = PQ_ERR_EPILOGUE;
    const int quarter = warp & 3, side = (warp - 20) >> 2;
    const int channel = 32 * quarter + lane, in_strip = channel & 15;
    const uint32_t from = tmem + kAColumns + (static_cast<uint32_t>(32 * quarter) << 16) + (kSplit ? side * kCols : 0);
    const uint32_t scale_in = w_base + (channel >> 4) * w.block_bytes + 1024 + ((in_strip & 7) * 2 + (in_strip >> 3)) * w.s_bytes;
    const uint32_t exchange = w_base + kStages * kWBytes;
    const int jobs = kbs * kPerStage;  // of a tile
    float sum[kCols];
    wait_previous_kernel();  // before anything is written
    Ring r, place;
    int job = 0, slot = 0;  // over all tiles
    if (!kSplit && side == 1) {
      ++job, ++slot;
      place.next(kPlaces);
      if (kPerStage == 1) r.next(kStages);
    }
    bool ok = true;
    for (int t = first_tile, end = jobs; t < tiles; t += tile_step, end += jobs) {
#pragma unroll
      for (int j = 0; j < kCols; ++j) sum[j] = 0.0f;
      for (; ok && job < end; job += kSplit ? 1 : 2) {
        ok = __all_sync(0xffffffffu, mbar_wait(bars.acc_full(place.s), place.phase, ctx)) != 0;
        if (!ok) break;
        tc_fence_after();
        const int h = kPerStage == 1 ? 0 : kSplit ? job & 1 : side;
#pragma unroll
        for (int g = 0; g < kAccs; ++g) {
          // (channels past the last strip have no scale there; they are not written)
          const float s = scale_in_smem(scale_in + r.s * kWBytes + (h * kAccs + g) * 16 * w.s_bytes, w.s_type);
#pragma unroll
          for (int j = 0; j < kCols; j += 32) {
            uint32_t v[32];
            tmem_ld32(from + (place.s * kAccs + g) * BN + j, v);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; i += 2) fma_pair(sum[j + i], sum[j + i + 1], __uint_as_float(v[i]), __uint_as_float(v[i + 1]), s);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bars.acc_empty(place.s));
          mbar_arrive(bars.slot_empty(slot));
          mbar_arrive(bars.stage_empty(r.s));
        }
        place.next(kPlaces);
        if (kSplit) {
          slot = (slot + 1) & (kSlots - 1);
          if (kPerStage == 1 || (job & 1)) r.next(kStages);
        } else {
          place.next(kPlaces);
          slot = (slot + 2) & (kSlots - 1);
          r.next(kStages);
          if (kPerStage == 1) r.next(kStages);
        }
      }
      if (p.k_parts > 1) break;  // (its only tile)
      int n_tile;
      int64_t m0;
      tile_origin(p, t, BN, &n_tile, &m0);
      const int n = n_tile * 128 + channel;
      if (!kSplit) {
        // each side writes half of the tokens: the other half's sums go to the other side.  (Every warp comes here for every tile, even
        // after a wait that ran out.)
#pragma unroll
        for (int j = 0; j < BN / 2; ++j)
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(exchange + ((side * (BN / 2) + j) * 128 + channel) * 4),
                       "f"(side == 0 ? sum[BN / 2 + j] : sum[j])
                       : "memory");
        asm volatile("bar.sync 1, 256;" ::: "memory");
#pragma unroll
        for (int j = 0; j < BN / 2; ++j) {
          float other;
          asm volatile("ld.shared.f32 %0, [%1];" : "=f"(other) : "r"(exchange + (((1 - side) * (BN / 2) + j) * 128 + channel) * 4) : "memory");
          sum[j] = side == 0 ? sum[j] + other : other + sum[BN / 2 + j];
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
      }
      if (ok && n < p.a.N) {
        const float bias = p.a.bias != nullptr ? p.a.bias[n] : 0.0f;
        const int64_t m = m0 + side * (BN / 2);
        const int left = static_cast<int>(min(static_cast<int64_t>(BN / 2), p.a.M - m));
#pragma unroll
        for (int j = 0; j < BN / 2; ++j)
          if (j < left) put_w4(p.a, m + j, n, p.a.bias != nullptr ? sum[j] + bias : sum[j]);
      }
    }
    if (p.k_parts > 1) {
      // Add the cluster's parts: every block writes a share of the tokens, a warp 32 channels of one at a time.  The ring is idle:
      // this block's only tile is over, but for the other side's last slot, which reads no tokens.
      asm volatile("bar.sync 1, 256;" ::: "memory");
      constexpr int kSides = kSplit ? 1 : 2;
#pragma unroll
      for (int j = 0; j < kCols; ++j)
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(tok_base + ((side * kCols + j) * 128 + channel) * 4), "f"(sum[j]) : "memory");
      int n_tile;
      int64_t m0;
      tile_origin(p, first_tile, BN, &n_tile, &m0);
      const int n = n_tile * 128 + channel;
      const float bias = p.a.bias != nullptr && n < p.a.N ? p.a.bias[n] : 0.0f;
      cluster_sync();
      const int j1 = static_cast<int>(min(static_cast<int64_t>(BN * (rank + 1) / p.k_parts), p.a.M - m0));
      if (ok)
        for (int j0 = BN * rank / p.k_parts + side; j0 < j1; j0 += 2 * kJoin) {
          // (kJoin tokens' loads from a peer on their way together)
          float y[kJoin] = {};
          for (int b = 0; b < p.k_parts; ++b) {
            float v[kSides][kJoin];
#pragma unroll
            for (int i = 0; i < kJoin; ++i)
#pragma unroll
              for (int s = 0; s < kSides; ++s)
                v[s][i] = j0 + 2 * i < j1 ? load_of_peer_f32(tok_base + ((s * BN + j0 + 2 * i) * 128 + channel) * 4, b) : 0.0f;
#pragma unroll
            for (int i = 0; i < kJoin; ++i)
#pragma unroll
              for (int s = 0; s < kSides; ++s) y[i] += v[s][i];
          }
#pragma unroll
          for (int i = 0; i < kJoin; ++i)
            if (n < p.a.N && j0 + 2 * i < j1) put_w4(p.a, m0 + j0 + 2 * i, n, p.a.bias != nullptr ? y[i] + bias : y[i]);
        }
      cluster_sync();
    }
  }
  // the blocks of a cluster leave together: their sums are read by the others
  if (p.k_parts > 1 && (warp < 20 || warp >= 28)) {
    cluster_sync();
    cluster_sync();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

template <typename T, int BN, int GS, int PARTS>
cudaError_t launch(const W4Tc& p, const CUtensorMap& x, int sms, bool after_copy, cudaStream_t stream) {
  static int attr_set[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(pq_linear_w4_tc<T, BN, GS, PARTS>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes(BN, PARTS));
    if (e != cudaSuccess) return e;
    if (dev < 64) attr_set[dev] = 1;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem_bytes(BN, PARTS);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(p.k_parts);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = after_copy ? 2 : 1;
  const int64_t tiles = static_cast<int64_t>(p.n_tiles) * p.m_tiles;
  // a cluster that shares K has one tile; otherwise as many blocks as there are SMs take the tiles in turn
  const int64_t at_once = p.k_parts > 1 ? tiles : std::min<int64_t>(tiles, sms);
  cfg.gridDim = dim3(static_cast<unsigned>(at_once * p.k_parts));
  return cudaLaunchKernelEx(&cfg, pq_linear_w4_tc<T, BN, GS, PARTS>, p, x);
}

template <typename T, int BN, int PARTS>
cudaError_t launch_group(const W4Tc& p, const CUtensorMap& x, int sms, bool after_copy, cudaStream_t s) {
  const int gs = p.a.p.group_shift;
  if constexpr (BN < 128)
    if (gs == 5) return launch<T, BN, 5, PARTS>(p, x, sms, after_copy, s);
  return gs == 6 ? launch<T, BN, 6, PARTS>(p, x, sms, after_copy, s) : launch<T, BN, 7, PARTS>(p, x, sms, after_copy, s);
}

template <typename T>
cudaError_t launch_bn(const W4Tc& p, int bn, const CUtensorMap& x, int sms, bool after_copy, cudaStream_t s) {
  return bn == 32   ? launch_group<T, 32, 1>(p, x, sms, after_copy, s)
         : bn == 64 ? launch_group<T, 64, 1>(p, x, sms, after_copy, s)
                    : launch_group<T, 128, 1>(p, x, sms, after_copy, s);
}

// ------------------------------------------------------------------ the tokens' copy
// Tokens that the tensor cores cannot load where they are: 16-bit ones in rows off 16-byte boundaries, and fp32 ones as three parts,
// into rows of `pitch` elements (zeros past K), a part below the other.  Bound by the launch; a thread four elements.
template <typename T>
__global__ void __launch_bounds__(256) pq_w4_tokens(const T* __restrict__ x, int64_t ldx, int64_t M, int K, uint16_t* __restrict__ out, int64_t pitch, bool wide) {
  let_next_kernel_start();
  const int64_t pieces = pitch / 4, total = M * pieces;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t m = i / pieces;
    const int k = static_cast<int>(i - m * pieces) * 4;
    T v[4];
    load4(x + m * ldx + min(k, K - 1), K - k, wide, v);
    uint32_t y[kParts<T>][2];
    operand_pairs(v, y);
#pragma unroll
    for (int part = 0; part < kParts<T>; ++part)
      *reinterpret_cast<uint2*>(out + (part * M + m) * pitch + k) = make_uint2(y[part][0], y[part][1]);
  }
}

template <typename T>
cudaError_t launch_tokens(const W4Args& a, uint16_t* out, int64_t pitch, cudaStream_t s) {
  const int64_t blocks = (a.M * (pitch / 4) + 255) / 256;
  pq_w4_tokens<T><<<static_cast<unsigned>(std::min<int64_t>(blocks, 152 * 16)), 256, 0, s>>>(static_cast<const T*>(a.x), a.ldx, a.M, a.K, out, pitch, a.wide_x);
  return cudaGetLastError();
}

}  // namespace

// From 17 tokens on, fp32 from 9; not where the kernel for few tokens is over in the 7 to 9 us that this one takes at least (us in a graph,
// here against there, N x K: bf16, 20 tokens: 1024 x 1024 7.9 / 6.5, 1024 x 2048 8.5 / 11.3, 8192 x 512 7.1 / 11.8, 4096 x 4096 11.0 / 28.6;
// 60 tokens: 1024 x 1024 9.7 / 8.0, 2048 x 2048 10.9 / 14.7; 16 tokens: 8192 x 4096 14.2 / 10.7; fp32, 12 tokens: 1024 x 1024 9.2 / 6.2,
// 2048 x 2048 9.6 / 16.2; 60 tokens: 1024 x 1024 9.4 / 11.2).
static bool worth(int64_t M, int N, int K, int x_type) {
  const int64_t rows = x_type == PQ_F32 ? 16 : 32;  // that the other kernel takes at one time
  return M > (x_type == PQ_F32 ? 8 : 16) && M <= (1 << 29) && (K > 1024 || (M + rows - 1) / rows * static_cast<double>(N) * K >= 4e6);
}

size_t w4_tc_scratch(int64_t M, int N, int K, int64_t ldx, int x_type) {
  if (!worth(M, N, K, x_type) || (x_type != PQ_F32 && ldx % 8 == 0)) return 0;
  return static_cast<size_t>(M) * static_cast<size_t>((K + 7) / 8 * 8) * 2 * (x_type == PQ_F32 ? 3 : 1);
}

bool w4_tc_takes(const W4Args& a, int x_type) {
  return worth(a.M, a.N, a.K, x_type) && (x_type == PQ_F32 || a.ldx % 8 != 0 || is_aligned(a.x, 16));
}

cudaError_t launch_w4_tc(const W4Args& given, int x_type, void* scratch, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  W4Tc p = {};
  p.a = given;
  p.err = device_error_word();
  p.wait_limit_ns = wait_limit_ns();
  if (p.err == nullptr) return cudaErrorInitializationError;
  W4Args& a = p.a;
  const bool copy = w4_tc_scratch(a.M, a.N, a.K, a.ldx, x_type) > 0;
  const int parts = x_type == PQ_F32 ? 3 : 1;
  // (groups of 32 have two accumulators for each 64 of K: the tensor memory holds those of two jobs of 64 tokens, not of 128; three
  // parts of 32 tokens are as many bytes as 96)
  const int bn = a.M <= 32 || parts == 3 ? 32 : a.M <= 64 || a.p.group_shift == 5 ? 64 : 128;
  p.n_tiles = (a.p.strips + kTileStrips - 1) / kTileStrips;
  const int64_t m_tiles = (a.M + bn - 1) / bn;
  if (p.n_tiles * m_tiles > 0x7FFFFFFF) return cudaErrorInvalidValue;
  p.m_tiles = static_cast<int>(m_tiles);
  // the blocks of a cluster share K while the chip has room for them and each keeps 512 of K
  p.k_parts = 1;
  for (int c = 2; c <= 8 && p.n_tiles * m_tiles * c <= (c == 8 ? sms / 2 : sms) && a.p.blocks / c >= 4; c *= 2) p.k_parts = c;
  if (copy) {
    const int64_t pitch = (a.K + 7) / 8 * 8;
    uint16_t* out = static_cast<uint16_t*>(scratch);
    e = x_type == PQ_F32   ? launch_tokens<float>(a, out, pitch, stream)
        : x_type == PQ_F16 ? launch_tokens<__half>(a, out, pitch, stream)
                           : launch_tokens<__nv_bfloat16>(a, out, pitch, stream);
    if (e != cudaSuccess) return e;
    a.x = scratch;
    a.ldx = pitch;
  }
  CUtensorMap x;
  if (!encode_map_2d(&x, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, a.x, static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.M) * parts,
                     static_cast<uint64_t>(a.ldx) * 2, 64, static_cast<uint32_t>(bn), CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorInvalidValue;
  if (parts == 3) return launch_group<__nv_bfloat16, 32, 3>(p, x, sms, copy, stream);
  return x_type == PQ_F16 ? launch_bn<__half>(p, bn, x, sms, copy, stream) : launch_bn<__nv_bfloat16>(p, bn, x, sms, copy, stream);
}

}  // namespace pq
