// Dense layer on 8-bit codes for many tokens, on the 5th-generation tensor cores.
//
// Mathematics.  acc[m, n] = sum_k q[m, k] w[n, k], exact.  sm_103a has no 8-bit integer
// tcgen05 kind (and mma.sync on 8-bit integers runs at 158 TOPS), but 8-bit codes
// are exact half values: kind::f16 multiplies them exactly and its fp32 sums of
// integers stay exact below 2^24, that is for 1024 of K (127 * 128 * 1024 < 2^24).  Every
// 1024 of K the sums move from tensor memory into int32 registers.
//
// Tile.  128 output channels (the MMA's rows) x BN tokens (its columns).  The weights stay
// 8-bit in memory: four warps turn each 128 x 64 block into halves and put it into
// tensor memory, from where the MMA takes its first operand, so the halves cost neither
// memory traffic nor shared-memory bandwidth.  The tokens come as halves
// (PQ_CODES_F16, written by the token quantiser) by TMA, in the 128-byte swizzle that
// the MMA reads.  Bound by the tensor rate for many tokens, by the weights' bytes for few.
//
// Drain.  Two accumulators take turns, so that one is read while the other is
// written: with 256 tokens they are the tile's two halves, and the issue order runs two
// K blocks of the first half, then the same two of the second, which leaves the
// first half's drain the time of two K blocks; with fewer tokens they alternate
// from one 1024-wide stretch (or tile) to the next.
//
// Roles (16 warps): 0 loads, 1 issues the MMAs, 4-7 convert, 8-15 drain and write.
// Few tiles: the blocks of a cluster take parts of K of one tile and add their
// int32 sums through distributed shared memory (in a fixed order; exact anyway).
#include <cuda_runtime.h>

#include <algorithm>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_linear.h"
#include "pq_tokens.cuh"

namespace pq {
namespace {

constexpr int kTcThreads = 512;
constexpr int kTcBK = 64;           // K of one stage: 64 bytes of a weight row, 128 of a token row
constexpr int kTcExact = 16;        // stages whose fp32 sums are exact
constexpr int kTcWBytes = 128 * kTcBK;
constexpr int kTcMaxStages = 8;

struct TcShape {
  int halves, nb, stages;  // accumulators of one tile, their columns, stages of the ring
};
__host__ __device__ constexpr TcShape tc_shape(int BN) {
  return BN == 256 ? TcShape{2, 128, 5} : TcShape{1, BN, 8};
}
__host__ __device__ constexpr int tc_smem(int BN) {
  return tc_shape(BN).stages * (kTcWBytes + BN * 128) + 1024 /* alignment */ + 512 /* barriers */;
}

// Barriers, 8 bytes each: w_full, b_full, a_full, empty (a ring each), acc_full,
// acc_empty (two each), done.
struct TcBars {
  uint32_t base;
  __device__ uint32_t w_full(int s) const { return base + 8u * s; }
  __device__ uint32_t b_full(int s) const { return base + 8u * (kTcMaxStages + s); }
  __device__ uint32_t a_full(int s) const { return base + 8u * (2 * kTcMaxStages + s); }
  __device__ uint32_t empty(int s) const { return base + 8u * (3 * kTcMaxStages + s); }
  __device__ uint32_t acc_full(int i) const { return base + 8u * (4 * kTcMaxStages + i); }
  __device__ uint32_t acc_empty(int i) const { return base + 8u * (4 * kTcMaxStages + 2 + i); }
  __device__ uint32_t done() const { return base + 8u * (4 * kTcMaxStages + 4); }
};

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void* tmap, int c0, int c1, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(bar)
      : "memory");
}

// K-major operand in the 128-byte swizzle: rows of 128 bytes, groups of 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t sw128_desc(uint32_t addr) {
  return static_cast<uint64_t>((addr >> 4) & 0x3FFFu) | (static_cast<uint64_t>(1) << 16) |
         (static_cast<uint64_t>(1024 >> 4) << 32) | (static_cast<uint64_t>(1) << 46) | (static_cast<uint64_t>(2) << 61);
}

// Instruction descriptor of kind::f16: half operands, fp32 sums, K-major, M = 128.
__host__ __device__ constexpr uint32_t idesc_f16_f32(int N) {
  return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(128 >> 4) << 24);
}

// Four MMAs (64 of K) with the first operand in tensor memory; the whole warp calls, one lane issues.
__device__ __forceinline__ void tc_mma_f16_ts_x4(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p, q, e;\nelect.sync _|e, 0xffffffff;\nsetp.ne.b32 p, %10, 0;\nsetp.eq.b32 q, 0, 0;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %5, %9, p;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%2], %6, %9, q;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%3], %7, %9, q;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%4], %8, %9, q;\n}" ::"r"(d),
      "r"(a), "r"(a + 8), "r"(a + 16), "r"(a + 24), "l"(b), "l"(b + 2), "l"(b + 4), "l"(b + 6), "r"(idesc), "r"(accumulate)
      : "memory");
}

// 32 columns of this warp's 32 tensor-memory lanes.
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ int32_t load_of_peer(uint32_t addr, uint32_t rank) {
  uint32_t a;
  int32_t v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}

// Position in the ring.
struct Ring {
  int s = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int stages) {
    if (++s == stages) s = 0, phase ^= 1u;
  }
};

// Tile t: channel tiles in bands of 16, the tokens' tiles along a band, so that the
// tiles at work at one time share weights and tokens in L2.
__device__ __forceinline__ void tile_origin(const LinearTc& p, int t, int BN, int* n0, int64_t* m0) {
  const int band = t / (16 * p.m_tiles), in = t - band * 16 * p.m_tiles;
  const int width = min(16, p.n_tiles - band * 16);
  *n0 = (band * 16 + in % width) * 128;
  *m0 = static_cast<int64_t>(in / width) * BN;
}

template <int BN>
__global__ void __launch_bounds__(kTcThreads, 1)
    pq_linear_tc(const __grid_constant__ LinearTc p, const __grid_constant__ CUtensorMap map_w,
                 const __grid_constant__ CUtensorMap map_q) {
  constexpr TcShape kS = tc_shape(BN);
  constexpr int kCols = kS.nb / 2;  // columns of an accumulator that one of its two draining warps takes
  constexpr uint32_t kABase = 256;  // first tensor-memory column of the weights' stages
  static_assert(2 * kS.nb <= 256 && 256 + 32 * kS.stages <= 512, "tensor memory");
  extern __shared__ uint8_t raw[];
  __shared__ int abort_flag;
  __shared__ uint32_t tmem_base;
  const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
  const uint32_t tok_base = smem, w_base = smem + kS.stages * BN * 128u;
  const TcBars bars{w_base + kS.stages * kTcWBytes};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kS.stages; ++s) {
      mbar_init(bars.w_full(s), 1);
      mbar_init(bars.b_full(s), 1);
      mbar_init(bars.a_full(s), 4);
      mbar_init(bars.empty(s), 1);
    }
    for (int i = 0; i < 2; ++i) {
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
  const int all = (p.a.K + kTcBK - 1) / kTcBK;
  const int rank = p.k_parts > 1 ? static_cast<int>(cluster_rank()) : 0;
  const int kb0 = static_cast<int>(static_cast<int64_t>(all) * rank / p.k_parts);
  const int kbs = static_cast<int>(static_cast<int64_t>(all) * (rank + 1) / p.k_parts) - kb0;
  const int first_tile = blockIdx.x / p.k_parts, tile_step = gridDim.x / p.k_parts;
  const int tiles = p.n_tiles * p.m_tiles;
  WaitCtx ctx{&abort_flag, p.err, p.wait_limit_ns, PQ_ERR_PRODUCER};

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0 && lane == 0) {
      // ---- loads.  The weights do not depend on the kernel before this one.
      Ring r;
      int issued = 0;
      int n0;
      int64_t m0;
      tile_origin(p, first_tile, BN, &n0, &m0);
      const int ahead = first_tile < tiles ? min(kS.stages, kbs) : 0;
      auto load_w = [&](int s, int kb) {
        mbar_arrive_expect_tx(bars.w_full(s), kTcWBytes);
        tma_load_2d(w_base + s * kTcWBytes, &map_w, (kb0 + kb) * kTcBK, n0, bars.w_full(s));
      };
      for (int i = 0; i < ahead; ++i) load_w(i, i);
      wait_previous_kernel();
      bool ok = true;
      int total = 0;
      for (int t = first_tile; ok && t < tiles; t += tile_step) {
        tile_origin(p, t, BN, &n0, &m0);
        for (int kb = 0; kb < kbs; ++kb, ++total) {
          if (total >= kS.stages && !mbar_wait(bars.empty(r.s), r.phase ^ 1u, ctx)) {
            ok = false;
            break;
          }
          if (total >= ahead) load_w(r.s, kb);
          mbar_arrive_expect_tx(bars.b_full(r.s), BN * 128);
          tma_load_2d(tok_base + r.s * BN * 128, &map_q, (kb0 + kb) * kTcBK, static_cast<int>(m0), bars.b_full(r.s));
          ++issued;
          r.next(kS.stages);
        }
      }
      // what was loaded last may still be on its way (all of `ahead` was issued)
      const int w_issued = max(issued, ahead);
      for (int k = max(0, w_issued - kS.stages); k < w_issued; ++k)
        mbar_wait_drain(bars.w_full(k % kS.stages), (k / kS.stages) & 1, p.wait_limit_ns, p.err);
      for (int k = max(0, issued - kS.stages); k < issued; ++k)
        mbar_wait_drain(bars.b_full(k % kS.stages), (k / kS.stages) & 1, p.wait_limit_ns, p.err);
    } else if (warp == 1) {
      // ---- MMAs
      ctx.err_bits = PQ_ERR_MMA;
      constexpr uint32_t idesc = idesc_f16_f32(kS.nb);
      auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, ctx)); };
      Ring r;
      uint32_t stretch = 0;  // exact stretches of K so far, over all tiles
      bool ok = true;
      for (int t = first_tile; ok && t < tiles; t += tile_step) {
        for (int c0 = 0; ok && c0 < kbs; c0 += kTcExact) {
          const int c1 = min(kbs, c0 + kTcExact);
          // times that this stretch's accumulators were used before
          const uint32_t uses = kS.halves == 2 ? stretch : stretch >> 1;
          for (int g0 = c0; ok && g0 < c1; g0 += 2) {
            const int g1 = min(c1, g0 + 2);
            const Ring start = r;
#pragma unroll
            for (int h = 0; h < kS.halves; ++h) {
              const int buf = kS.halves == 2 ? h : stretch & 1;
              Ring x = start;
              for (int kb = g0; kb < g1; ++kb) {
                if (kb == c0 && uses > 0) ok = ok && wait(bars.acc_empty(buf), (uses - 1) & 1);
                if (h == 0) ok = ok && wait(bars.a_full(x.s), x.phase) && wait(bars.b_full(x.s), x.phase);
                if (!ok) break;
                tc_fence_after();
                tc_mma_f16_ts_x4(tmem + buf * kS.nb, tmem + kABase + 32 * x.s,
                                 sw128_desc(tok_base + x.s * BN * 128 + h * 128 * 128), idesc, kb != c0);
                if (h == kS.halves - 1) tc_commit_warp(bars.empty(x.s));
                x.next(kS.stages);
              }
              if (!ok) break;
              if (g1 == c1) tc_commit_warp(bars.acc_full(buf));
              r = x;
            }
          }
          ++stretch;
        }
      }
      // every MMA issued must be over before the tensor memory is given back
      tc_commit_warp(bars.done());
      if (lane == 0) mbar_wait_drain(bars.done(), 0, p.wait_limit_ns, p.err);
      __syncwarp();
    }
  } else if (warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    // ---- weights to halves: this thread's row of each block
    ctx.err_bits = PQ_ERR_EPILOGUE;
    const int row = 32 * (warp - 4) + lane;
    const uint32_t swizzle = (row >> 1) & 3;
    const uint32_t lanes = static_cast<uint32_t>(32 * (warp - 4)) << 16;
    Ring r;
    bool ok = true;
    for (int t = first_tile; ok && t < tiles; t += tile_step)
      for (int kb = 0; kb < kbs; ++kb) {
        ok = __all_sync(0xffffffffu, mbar_wait(bars.w_full(r.s), r.phase, ctx));
        if (!ok) break;
        const uint32_t src = w_base + r.s * kTcWBytes + row * kTcBK;
        uint32_t h[32];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 v = lds128(src + ((i ^ swizzle) << 4));
          half_of_codes(v.x, h[8 * i], h[8 * i + 1]);
          half_of_codes(v.y, h[8 * i + 2], h[8 * i + 3]);
          half_of_codes(v.z, h[8 * i + 4], h[8 * i + 5]);
          half_of_codes(v.w, h[8 * i + 6], h[8 * i + 7]);
        }
        tmem_st32(tmem + lanes + kABase + 32 * r.s, h);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bars.a_full(r.s));
        r.next(kS.stages);
      }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
    // ---- sums and outputs: this thread's channel, half of each accumulator's tokens
    ctx.err_bits = PQ_ERR_EPILOGUE;
    const int quarter = warp & 3, side = (warp - 8) >> 2;
    const uint32_t from = tmem + (static_cast<uint32_t>(32 * quarter) << 16) + side * kCols;
    wait_previous_kernel();  // the tokens' scales
    int32_t sum[kS.halves][kCols];
    uint32_t stretch = 0;
    bool ok = true;
    for (int t = first_tile; ok && t < tiles; t += tile_step) {
#pragma unroll
      for (int h = 0; h < kS.halves; ++h)
#pragma unroll
        for (int j = 0; j < kCols; ++j) sum[h][j] = 0;
      for (int c0 = 0; ok && c0 < kbs; c0 += kTcExact) {
#pragma unroll
        for (int h = 0; h < kS.halves; ++h) {
          const int buf = kS.halves == 2 ? h : stretch & 1;
          const uint32_t uses = kS.halves == 2 ? stretch : stretch >> 1;
          ok = ok && __all_sync(0xffffffffu, mbar_wait(bars.acc_full(buf), uses & 1, ctx));
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int j = 0; j < kCols; j += 16) {
            uint32_t v[16];
            tmem_ld16(from + buf * kS.nb + j, v);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[h][j + i] += __float2int_rn(__uint_as_float(v[i]));
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bars.acc_empty(buf));
        }
        ++stretch;
      }
      if (!ok) break;
      if (p.k_parts > 1) {
        // the ring is idle: this block's only tile is over (the last accumulator was full)
        if (BN <= 128) {
#pragma unroll
          for (int j = 0; j < kCols; ++j)
            asm volatile("st.shared.s32 [%0], %1;" ::"r"(tok_base + ((side * kCols + j) * 128 + 32 * quarter + lane) * 4),
                         "r"(sum[0][j])
                         : "memory");
        }
        break;
      }
      int n0;
      int64_t m0;
      tile_origin(p, t, BN, &n0, &m0);
      const int n = n0 + 32 * quarter + lane;
      if (n < p.a.N) {
        const float s_w = p.a.s_w != nullptr ? p.a.s_w[n] : 0.0f, bias = p.a.bias != nullptr ? p.a.bias[n] : 0.0f;
#pragma unroll
        for (int h = 0; h < kS.halves; ++h) {
          const int64_t m = m0 + h * 128 + side * kCols;
#pragma unroll
          for (int j = 0; j < kCols; ++j)
            if (m + j < p.a.M) put_result(p.a, m + j, n, sum[h][j], s_w, bias);
        }
      }
    }
    if (p.k_parts > 1) {
      // add the cluster's parts: every block writes a share of the tokens
      cluster_sync();
      int n0;
      int64_t m0;
      tile_origin(p, first_tile, BN, &n0, &m0);
      const int c = threadIdx.x & 127, n = n0 + c;
      const int j0 = BN * rank / p.k_parts, j1 = BN * (rank + 1) / p.k_parts;
      if (ok && n < p.a.N) {
        const float s_w = p.a.s_w != nullptr ? p.a.s_w[n] : 0.0f, bias = p.a.bias != nullptr ? p.a.bias[n] : 0.0f;
        for (int j = j0 + side; j < j1 && m0 + j < p.a.M; j += 2) {
          int32_t acc = 0;
          for (int b = 0; b < p.k_parts; ++b) acc += load_of_peer(tok_base + (j * 128 + c) * 4, b);
          put_result(p.a, m0 + j, n, acc, s_w, bias);
        }
      }
      cluster_sync();
    }
  }
  // the blocks of a cluster leave together: their sums are read by the others
  if (p.k_parts > 1 && warp < 8) {
    cluster_sync();
    cluster_sync();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int BN>
cudaError_t launch(const LinearTc& p, const CUtensorMap& w, const CUtensorMap& q, int grid, bool after_tokens,
                   cudaStream_t stream) {
  static int attr_set[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(pq_linear_tc<BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, tc_smem(BN));
    if (e != cudaSuccess) return e;
    if (dev < 64) attr_set[dev] = 1;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(kTcThreads);
  cfg.dynamicSmemBytes = tc_smem(BN);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (after_tokens) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (p.k_parts > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = static_cast<unsigned>(p.k_parts);
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, pq_linear_tc<BN>, p, w, q);
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
  p.n_tiles = (a.N + 127) / 128;
  auto tiles_of = [&](int bn) { return static_cast<int64_t>(p.n_tiles) * ((a.M + bn - 1) / bn); };
  auto cost = [&](int bn) { return (tiles_of(bn) + sms - 1) / sms * bn; };
  // tokens of a tile: the fewest that hold all of them, beyond 128 what leaves the
  // last round of tiles the fullest
  const int bn = a.M <= 32 ? 32 : a.M <= 64 ? 64 : a.M <= 128 ? 128 : cost(128) < cost(256) ? 128 : 256;
  p.m_tiles = static_cast<int>((a.M + bn - 1) / bn);
  const int64_t tiles = tiles_of(bn);
  if (tiles > 0x7FFFFFFF) return cudaErrorInvalidValue;
  // parts of K: while the chip is less than half full and each part keeps 256 of K
  p.k_parts = 1;
  while (bn <= 128 && p.k_parts < 8 && tiles * p.k_parts * 2 <= sms && a.K / (p.k_parts * 2) >= 256) p.k_parts *= 2;
  const int grid = p.k_parts > 1 ? static_cast<int>(tiles) * p.k_parts : static_cast<int>(std::min<int64_t>(tiles, sms));
  CUtensorMap w, q;
  if (!encode_map_2d(&w, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.w, static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.N),
                     static_cast<uint64_t>(a.ldw), kTcBK, 128, CU_TENSOR_MAP_SWIZZLE_64B) ||
      !encode_map_2d(&q, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, a.q, static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.M),
                     static_cast<uint64_t>(a.ldq) * 2, kTcBK, static_cast<uint32_t>(bn), CU_TENSOR_MAP_SWIZZLE_128B))
    return cudaErrorInvalidValue;
  if (bn == 32) return launch<32>(p, w, q, grid, after_tokens, stream);
  if (bn == 64) return launch<64>(p, w, q, grid, after_tokens, stream);
  if (bn == 128) return launch<128>(p, w, q, grid, after_tokens, stream);
  return launch<256>(p, w, q, grid, after_tokens, stream);
}

}  // namespace pq
