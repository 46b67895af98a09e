// Dense layers with 4-bit weights for a batch of tokens, on the 5th-generation tensor cores.
//
// Mathematics.  For each group of input channels, kind::f16 multiplies the codes (integers, exact in the activations' type) with
// the activations into an accumulator of its own, in fp32; it is read back, multiplied with the channel's scale of the group and
// added in registers, in fp32.  So a weight is never rounded: scaled to 16 bits before the product it would be, by as much as the
// output is.
//
// Tile.  128 output channels (8 packed strips) x BN tokens a block.  Codes stay 4-bit in memory and shared memory; eight warps turn
// them into 16-bit operands in tensor memory, which take no shared-memory bandwidth: a lane's packed 16 bytes are, unpacked, the
// registers of a 16 x 256-bit store, so nothing is exchanged between lanes.  Activations come by TMA in the 128-byte swizzle.
// The accumulators of groups take turns, so that one is read while others are written.  Few tiles: the blocks of a cluster take
// parts of K of one tile and add their fp32 sums through distributed shared memory, in order.
//
// Roles (20 warps): 0 and 2 load (weights, tokens), 1 issues the MMAs, 4-7 and 8-11 unpack 64 of K each of every stage, 12-19 drain
// and write.  A stage is 128 of K.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_linear.h"
#include "pq_tc.cuh"
#include "pq_tokens.cuh"
#include "pq_w4.cuh"

namespace pq {
namespace {

constexpr int kThreads = 640;
constexpr int kStrips = 8;                            // of a tile
constexpr int kWBytes = kStrips * (1024 + 256);       // of a stage's weights at most
constexpr int kMaxStages = 8;
constexpr int kSlots = 8;                             // 64 of K of unpacked weights each, 32 columns of tensor memory
constexpr uint32_t kAccColumns = 256;                 // of the accumulators

__host__ __device__ constexpr int stage_bytes(int BN) { return kWBytes + BN * 256; }
__host__ __device__ constexpr int stages(int BN) { return 204800 / stage_bytes(BN) < kMaxStages ? 204800 / stage_bytes(BN) : kMaxStages; }
__host__ __device__ constexpr int smem_bytes(int BN) { return stages(BN) * stage_bytes(BN) + 1024 /* alignment */; }

struct W4Tc {
  W4Args a;
  int n_tiles, m_tiles;  // tiles of 128 channels, of BN tokens
  int k_parts;           // blocks of a cluster that share a tile's K (1: none)
  unsigned int* err;
  uint64_t wait_limit_ns;
};

// Barriers: loaded (a stage's bytes), empty (its MMAs are over and its scales read), full (a slot is unpacked), slot_empty (its
// MMAs are over), acc_full, acc_empty, done.
struct Bars {
  uint32_t base;
  __device__ uint32_t loaded(int s) const { return base + 8u * s; }
  __device__ uint32_t empty(int s) const { return base + 8u * (kMaxStages + s); }
  __device__ uint32_t full(int s) const { return base + 8u * (2 * kMaxStages + s); }
  __device__ uint32_t slot_empty(int s) const { return base + 8u * (2 * kMaxStages + kSlots + s); }
  __device__ uint32_t acc_full(int i) const { return base + 8u * (2 * kMaxStages + 2 * kSlots + i); }
  __device__ uint32_t acc_empty(int i) const { return base + 8u * (2 * kMaxStages + 2 * kSlots + 8 + i); }
  __device__ uint32_t done() const { return base + 8u * (2 * kMaxStages + 2 * kSlots + 16); }
};
constexpr int kBars = 2 * kMaxStages + 2 * kSlots + 17;

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

// 16 lanes x 32 columns: lane 4 g + t holds of lanes g and g + 8, for each 8 columns, columns 2 t and 2 t + 1.
__device__ __forceinline__ void tmem_st_16x256b_x4(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
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

template <typename T, int BN>
__global__ void __launch_bounds__(kThreads, 1) pq_linear_w4_tc(const __grid_constant__ W4Tc p, const __grid_constant__ CUtensorMap map_x) {
  constexpr int kStages = stages(BN);
  constexpr int kAccs = kAccColumns / BN;
  constexpr int kTok = BN * 128;   // bytes of 64 of K of the tokens
  constexpr int kCols = BN / 2;    // columns of an accumulator that one of its two draining warps takes
  constexpr int kStep = kCols % 32 == 0 ? 32 : 16;
  extern __shared__ uint8_t raw[];
  __shared__ alignas(8) uint64_t bar_words[kBars];
  __shared__ int abort_flag;
  __shared__ uint32_t tmem_base;
  const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t tok_base = smem, w_base = smem + kStages * 2 * kTok;
  const Bars bars{smem_u32(bar_words)};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = p.k_parts > 1 ? static_cast<int>(cluster_rank()) : 0;
  const PackedW4& w = p.a.p;

  if (warp == 2 && lane == 0) prefetch_tmap(&map_x);
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(bars.loaded(s), 2);
      mbar_init(bars.empty(s), 1 + 8);
    }
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(bars.full(s), 4);
      mbar_init(bars.slot_empty(s), 1);
    }
    for (int i = 0; i < kAccs; ++i) {
      mbar_init(bars.acc_full(i), 1);
      mbar_init(bars.acc_empty(i), 8);
    }
    mbar_init(bars.done(), 1);
    abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc(smem_u32(&tmem_base), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;

  // this block's part of K, in stages, and its tiles
  const int kb0 = static_cast<int>(static_cast<int64_t>(w.blocks) * rank / p.k_parts);
  const int kbs = static_cast<int>(static_cast<int64_t>(w.blocks) * (rank + 1) / p.k_parts) - kb0;
  const int first_tile = blockIdx.x / p.k_parts, tile_step = gridDim.x / p.k_parts;
  const int tiles = p.n_tiles * p.m_tiles;
  WaitCtx ctx{&abort_flag, p.err, p.wait_limit_ns, PQ_ERR_PRODUCER};

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if ((warp == 0 || warp == 2) && lane == 0) {
      // ---- loads: a stage's strips (warp 0), its tokens (warp 2)
      const bool weights = warp == 0;
      Ring r;
      bool ok = true;
      int issued = 0;
      for (int t = first_tile; ok && t < tiles; t += tile_step) {
        int n_tile;
        int64_t m0;
        tile_origin(p, t, BN, &n_tile, &m0);
        const int strips = min(kStrips, w.strips - n_tile * kStrips);
        const uint8_t* from = p.a.w + n_tile * kStrips * w.strip_bytes() + static_cast<int64_t>(kb0) * w.block_bytes;
        for (int kb = 0; kb < kbs; ++kb, ++issued) {
          if (issued >= kStages && !mbar_wait(bars.empty(r.s), r.phase ^ 1u, ctx)) {
            ok = false;
            break;
          }
          const uint32_t bar = bars.loaded(r.s);
          if (weights) {
            mbar_arrive_expect_tx(bar, strips * w.block_bytes);
            for (int i = 0; i < strips; ++i)
              bulk_load(w_base + r.s * kWBytes + i * w.block_bytes, from + i * w.strip_bytes(), w.block_bytes, bar);
            from += w.block_bytes;
          } else {
            const int k = (kb0 + kb) * kBlockK;
            mbar_arrive_expect_tx(bar, 2 * kTok);
            tma_load_2d(tok_base + r.s * 2 * kTok, &map_x, k, static_cast<int>(m0), bar);
            tma_load_2d(tok_base + r.s * 2 * kTok + kTok, &map_x, k + 64, static_cast<int>(m0), bar);
          }
          r.next(kStages);
        }
      }
      // what was loaded last may still be on its way
      for (int k = max(0, issued - kStages); k < issued; ++k)
        mbar_wait_drain(bars.loaded(k % kStages), (k / kStages) & 1, p.wait_limit_ns, p.err);
    } else if (warp == 1) {
      // ---- MMAs
      ctx.err_bits = PQ_ERR_MMA;
      constexpr uint32_t idesc = idesc_of<T>(BN);
      auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, ctx)) != 0; };
      const int per_group = 1 << (w.group_shift - 5);  // MMA pairs of a group
      Ring r, slot, acc;
      uint32_t accs = 0;  // accumulators begun so far
      bool ok = true;
      for (int t = first_tile; ok && t < tiles; t += tile_step)
        for (int kb = 0; ok && kb < kbs; ++kb) {
          int in = 0;  // MMA pairs of the current group
          for (int h = 0; ok && h < 2; ++h) {
            ok = wait(bars.full(slot.s), slot.phase);
            if (!ok) break;
            tc_fence_after();
            for (int c = 0; c < 2; ++c) {
              if (in == 0 && accs >= kAccs) {
                ok = wait(bars.acc_empty(acc.s), acc.phase ^ 1u);
                if (!ok) break;
                tc_fence_after();
              }
              if (in == 0) ++accs;
              mma_ts_x2(tmem + acc.s * BN, tmem + kAccColumns + 32 * slot.s + 16 * c,
                        sw128_desc(tok_base + (2 * r.s + h) * kTok) + 4 * c, idesc, in > 0);
              if (++in == per_group) {
                tc_commit_warp(bars.acc_full(acc.s));
                acc.next(kAccs);
                in = 0;
              }
            }
            if (!ok) break;
            tc_commit_warp(bars.slot_empty(slot.s));
            slot.next(kSlots);
          }
          if (!ok) break;
          tc_commit_warp(bars.empty(r.s));
          r.next(kStages);
        }
      // every MMA issued must be over before the tensor memory is given back
      tc_commit_warp(bars.done());
      if (lane == 0) mbar_wait_drain(bars.done(), 0, p.wait_limit_ns, p.err);
      __syncwarp();
    }
  } else if (warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    // ---- codes to operands: this warp's 32 channels, 64 of K of every stage
    ctx.err_bits = PQ_ERR_EPILOGUE;
    const int quarter = warp & 3, half = (warp - 4) >> 2;
    const uint32_t to = tmem + kAccColumns + (static_cast<uint32_t>(32 * quarter) << 16);
    const int total = first_tile < tiles ? ((tiles - first_tile - 1) / tile_step + 1) * kbs : 0;
    Ring r;
    int slot = half;
    uint32_t round = 0;  // times that the slot was used before
    for (int i = 0; i < total; ++i) {
      if (!__all_sync(0xffffffffu, mbar_wait(bars.loaded(r.s), r.phase, ctx))) break;
      uint32_t h[2][16];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint4 v = lds128(w_base + r.s * kWBytes + (2 * quarter + j) * w.block_bytes + half * 512 + lane * 16);
        const uint32_t words[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t low = words[2 * (c >> 1)], high = words[2 * (c >> 1) + 1];  // rows g and g + 8
          if (c & 1) {
            h[j][4 * c] = code_pair<T, 2>(low), h[j][4 * c + 1] = code_pair<T, 3>(low);
            h[j][4 * c + 2] = code_pair<T, 2>(high), h[j][4 * c + 3] = code_pair<T, 3>(high);
          } else {
            h[j][4 * c] = code_pair<T, 0>(low), h[j][4 * c + 1] = code_pair<T, 1>(low);
            h[j][4 * c + 2] = code_pair<T, 0>(high), h[j][4 * c + 3] = code_pair<T, 1>(high);
          }
        }
      }
      if (round > 0 && !__all_sync(0xffffffffu, mbar_wait(bars.slot_empty(slot), (round - 1) & 1, ctx))) break;
      tc_fence_after();
      tmem_st_16x256b_x4(to + 32 * slot, h[0]);
      tmem_st_16x256b_x4(to + 32 * slot + (16u << 16), h[1]);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bars.full(slot));
      r.next(kStages);
      slot += 2;
      if (slot >= kSlots) slot = half, ++round;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 144;");
    // ---- sums and outputs: this thread's channel, half of each accumulator's tokens
    ctx.err_bits = PQ_ERR_EPILOGUE;
    const int quarter = warp & 3, side = (warp - 12) >> 2;
    const int channel = 32 * quarter + lane, in_strip = channel & 15;
    const uint32_t from = tmem + (static_cast<uint32_t>(32 * quarter) << 16) + side * kCols;
    const int per_block = kBlockK >> w.group_shift;  // groups of a stage
    const uint32_t scale_in = (channel >> 4) * w.block_bytes + 1024 + ((in_strip & 7) * 2 + (in_strip >> 3)) * w.s_bytes;
    float sum[kCols];
    Ring r, acc;
    bool ok = true;
    for (int t = first_tile; ok && t < tiles; t += tile_step) {
      int n_tile;
      int64_t m0;
      tile_origin(p, t, BN, &n_tile, &m0);
      const int n = n_tile * 128 + channel;
#pragma unroll
      for (int j = 0; j < kCols; ++j) sum[j] = 0.0f;
      for (int kb = 0; ok && kb < kbs; ++kb) {
        for (int g = 0; g < per_block; ++g) {
          ok = __all_sync(0xffffffffu, mbar_wait(bars.acc_full(acc.s), acc.phase, ctx)) != 0;
          if (!ok) break;
          tc_fence_after();
          // (channels past the last strip have no scale there; they are not written)
          const float s = scale_in_smem(w_base + r.s * kWBytes + scale_in + g * 16 * w.s_bytes, w.s_type);
#pragma unroll
          for (int j = 0; j < kCols; j += kStep) {
            uint32_t v[kStep];
            if constexpr (kStep == 32)
              tmem_ld32(from + acc.s * BN + j, v);
            else
              tmem_ld16(from + acc.s * BN + j, v);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < kStep; ++i) sum[j + i] = fmaf(s, __uint_as_float(v[i]), sum[j + i]);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bars.acc_empty(acc.s));
          acc.next(kAccs);
        }
        if (!ok) break;
        if (lane == 0) mbar_arrive(bars.empty(r.s));
        r.next(kStages);
      }
      if (!ok) break;
      if (p.k_parts > 1) {
        // the ring is idle: this block's only tile is over (the last accumulator was full)
#pragma unroll
        for (int j = 0; j < kCols; ++j)
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(tok_base + ((side * kCols + j) * 128 + channel) * 4), "f"(sum[j]) : "memory");
        break;
      }
      if (n < p.a.N) {
        const float bias = p.a.bias != nullptr ? p.a.bias[n] : 0.0f;
        const int left = static_cast<int>(min(static_cast<int64_t>(kCols), p.a.M - m0 - side * kCols));
#pragma unroll
        for (int j = 0; j < kCols; ++j)
          if (j < left) put_w4(p.a, m0 + side * kCols + j, n, p.a.bias != nullptr ? sum[j] + bias : sum[j]);
      }
    }
    if (p.k_parts > 1) {
      // add the cluster's parts: every block writes a share of the tokens, a warp 32 channels of one at a time
      int n_tile;
      int64_t m0;
      tile_origin(p, first_tile, BN, &n_tile, &m0);
      const int n = n_tile * 128 + channel;
      const float bias = p.a.bias != nullptr && n < p.a.N ? p.a.bias[n] : 0.0f;
      cluster_sync();
      const int j1 = static_cast<int>(min(static_cast<int64_t>(BN * (rank + 1) / p.k_parts), p.a.M - m0));
      if (ok)
        for (int j = BN * rank / p.k_parts + side; j < j1; j += 2) {
          float v[8];
#pragma unroll
          for (int b = 0; b < 8; ++b) v[b] = b < p.k_parts ? load_of_peer_f32(tok_base + (j * 128 + channel) * 4, b) : 0.0f;
          float y = v[0];
#pragma unroll
          for (int b = 1; b < 8; ++b) y += v[b];
          if (n < p.a.N) put_w4(p.a, m0 + j, n, p.a.bias != nullptr ? y + bias : y);
        }
      cluster_sync();
    }
  }
  // the blocks of a cluster leave together: their sums are read by the others
  if (p.k_parts > 1 && warp < 12) {
    cluster_sync();
    cluster_sync();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <typename T, int BN>
cudaError_t launch(const W4Tc& p, const CUtensorMap& x, int sms, cudaStream_t stream) {
  static int attr_set[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(pq_linear_w4_tc<T, BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes(BN));
    if (e != cudaSuccess) return e;
    if (dev < 64) attr_set[dev] = 1;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem_bytes(BN);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(p.k_parts);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const int64_t tiles = static_cast<int64_t>(p.n_tiles) * p.m_tiles;
  // a cluster that shares K has one tile; otherwise as many blocks as there are SMs take the tiles in turn
  const int64_t at_once = p.k_parts > 1 ? tiles : std::min<int64_t>(tiles, sms);
  cfg.gridDim = dim3(static_cast<unsigned>(at_once * p.k_parts));
  return cudaLaunchKernelEx(&cfg, pq_linear_w4_tc<T, BN>, p, x);
}

template <typename T>
cudaError_t launch_bn(const W4Tc& p, int bn, const CUtensorMap& x, int sms, cudaStream_t s) {
  return bn == 32 ? launch<T, 32>(p, x, sms, s) : bn == 64 ? launch<T, 64>(p, x, sms, s) : launch<T, 128>(p, x, sms, s);
}

}  // namespace

bool w4_tc_takes(const W4Args& a, int x_type) {
  return x_type != PQ_F32 && a.M > 8 && a.M <= (1 << 30) && is_aligned(a.x, 16) && a.ldx % 8 == 0;
}

cudaError_t launch_w4_tc(const W4Args& a, int x_type, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  W4Tc p = {};
  p.a = a;
  p.err = device_error_word();
  p.wait_limit_ns = wait_limit_ns();
  if (p.err == nullptr) return cudaErrorInitializationError;
  const int bn = a.M <= 32 ? 32 : a.M <= 64 ? 64 : 128;
  p.n_tiles = (a.p.strips + kStrips - 1) / kStrips;
  const int64_t m_tiles = (a.M + bn - 1) / bn;
  if (p.n_tiles * m_tiles > 0x7FFFFFFF) return cudaErrorInvalidValue;
  p.m_tiles = static_cast<int>(m_tiles);
  // the blocks of a cluster share K while the chip has room for them and each keeps 512 of K
  p.k_parts = 1;
  for (int c = 2; c <= 8 && p.n_tiles * m_tiles * c <= (c == 8 ? sms / 2 : sms) && a.p.blocks / c >= 4; c *= 2) p.k_parts = c;
  CUtensorMap x;
  if (!encode_map_2d(&x, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, a.x, static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.M),
                     static_cast<uint64_t>(a.ldx) * 2, 64, static_cast<uint32_t>(bn), CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorInvalidValue;
  return x_type == PQ_F16 ? launch_bn<__half>(p, bn, x, sms, stream) : launch_bn<__nv_bfloat16>(p, bn, x, sms, stream);
}

}  // namespace pq
