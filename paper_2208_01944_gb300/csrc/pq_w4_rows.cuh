// Dense layers with 4-bit weights for few tokens (and any alignment and type).  The mathematics is in linear_w4.cu.
#pragma once

#include <cuda_runtime.h>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_tokens.cuh"
#include "pq_w4.cuh"

namespace pq {
namespace {

// Rows g's and g + 8's scale of a group, neighbours in shared memory.
template <typename S>
__device__ __forceinline__ void scale_pair(uint32_t at, float& s0, float& s1) {
  if constexpr (sizeof(S) == 4) {
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(s0), "=f"(s1) : "r"(at) : "memory");
  } else {
    uint32_t w;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
    S s[2];
    memcpy(s, &w, 4);
    s0 = to_f32(s[0]), s1 = to_f32(s[1]);
  }
}

template <typename T>
__device__ __forceinline__ void mma_w4(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (sizeof(T) == 2 && !std::is_same<T, __nv_bfloat16>::value) {
    mma_16x8x16(d, a0, a1, a2, a3, b0, b1);
  } else {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
}

// A block: NS strips of 16 channels x 8 NT tokens; its warps take the strips' blocks of 128 of K in turn.  Bound by the weights'
// bytes and, close to it, by the instructions of unpacking.  The weights come through rings of asynchronous copies, one for each
// warp (a block of 128 of K a stage, kRing - 1 of them ahead); each lane reads codes that it copied itself, and scales that
// its warp copied (8 x 16384 x 8192, f16, groups of 128: 22 us, 3.1 TB/s; one x 4096 x 4096 5.0).  The tokens, which every block reads, come from L1 and L2 into registers, a block of K ahead
// where two fit; two strips share them (8 tokens' 128 of K are twice a strip's bytes).  The loop is unrolled over the ring, so that
// its places are constants (with one that was not, and the scales' type looked up, 128 of K of a strip took 218 instructions, not 176, and a
// token times 16384 x 8192 25 us, not 20).
constexpr int kWarps = 8;
constexpr int kPlace = 1024 + 256;  // bytes of 128 of K of a strip at most: four groups' fp32 scales

template <typename T, typename S, int NT, int NS, int kRing>
__global__ void __launch_bounds__(32 * kWarps) pq_linear_w4_rows(const __grid_constant__ W4Args a) {
  extern __shared__ __align__(16) uint8_t ring_raw[];
  __shared__ float part[kWarps][NS * NT][8][17];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * (8 * NT);
  const int strip = blockIdx.x * NS;
  const int bytes = a.p.block_bytes, pitch = a.p.pitch(strip);
  const int strips = min(NS, a.p.strips - strip);  // (neighbours in a tile)
  const uint8_t* from = a.w + a.p.strip_at(strip) + static_cast<int64_t>(warp) * pitch + lane * 16;
  const int64_t step = static_cast<int64_t>(kWarps) * pitch;
  const uint32_t ring = smem_u32(ring_raw) + warp * (kRing * NS * kPlace) + lane * 16;
  const uint32_t scales = smem_u32(ring_raw) + warp * (kRing * NS * kPlace) + 1024 + g * 2 * static_cast<uint32_t>(sizeof(S));
  const bool copies_scales = lane < (bytes - 1024) >> 4;
  const int mine = a.p.blocks > warp ? (a.p.blocks - warp - 1) / kWarps + 1 : 0;
  const int group_shift = a.p.group_shift;
  const uint32_t second_group = group_shift == 7 ? 0u : 64u >> group_shift;  // of the second 64 of K
  auto fetch = [&](int stage) {
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      if (n > 0 && n >= strips) break;
      const uint32_t to = ring + (stage * NS + n) * kPlace;
      const uint8_t* src = from + n * bytes;
      cp_async_16(to, src, 16);
      cp_async_16(to + 512, src + 512, 16);
      if (copies_scales) cp_async_16(to + 1024, src + 1024, 16);
    }
    from += step;
  };
#pragma unroll
  for (int i = 0; i < kRing - 1; ++i) {
    if (i < mine) fetch(i);
    cp_async_commit();
  }
  // Columns 128 b + 16 c + 4 t and up of a token.  (Tokens past the end read the tile's first again: their columns of the
  // products are not stored.)
  const T* row[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t m = m0 + 8 * j + g;
    row[j] = static_cast<const T*>(a.x) + (m < a.M ? m : m0) * a.ldx + 4 * t;
  }
  constexpr bool kWhole = NT * sizeof(T) <= 4;  // a block's tokens fit the registers
  constexpr bool kAhead = NT * sizeof(T) == 2;  // and so do the next one's
  const int whole_blocks = a.wide_x ? a.K / kBlockK : 0;  // those whose columns are all there, on boundaries of four
  struct Tokens {
    T v[NT][8][4];
  };
  auto load_tokens = [&](int i, Tokens& x) {
    const int b = warp + i * kWarps;
    if (b < whole_blocks) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int c = 0; c < 8; ++c) load4(row[j] + b * kBlockK + 16 * c, 4, true, x.v[j][c]);
    } else {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int c = 0; c < 8; ++c) load4(row[j] + b * kBlockK + 16 * c, a.K - (b * kBlockK + 16 * c + 4 * t), a.wide_x, x.v[j][c]);
    }
  };
  float sum[NS][NT][4] = {};
  auto multiply = [&](int i, int stage, const Tokens& x) {
    cp_async_wait<kRing - 2>();
    __syncwarp();  // the block's scales have arrived, and every lane is done with the stage before
    if (i + kRing - 1 < mine) fetch((stage + kRing - 1) % kRing);
    cp_async_commit();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        uint4 u;
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w)
                     : "r"(ring + (stage * NS + n) * kPlace + s * 512)
                     : "memory");
        const uint32_t words[4] = {u.x, u.y, u.z, u.w};
        float d[NT][4] = {};
        // a group of 32 is over, or 64 of K are (groups of 128: the same scale twice)
        auto scaled = [&](uint32_t group) {
          float s0, s1;
          scale_pair<S>(scales + (stage * NS + n) * kPlace + group * static_cast<uint32_t>(16 * sizeof(S)), s0, s1);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            sum[n][j][0] = fmaf(s0, d[j][0], sum[n][j][0]);
            sum[n][j][1] = fmaf(s0, d[j][1], sum[n][j][1]);
            sum[n][j][2] = fmaf(s1, d[j][2], sum[n][j][2]);
            sum[n][j][3] = fmaf(s1, d[j][3], sum[n][j][3]);
          }
        };
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t p[4], q[4];
          code_pairs<T>(words[2 * h], p);
          code_pairs<T>(words[2 * h + 1], q);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int in = 4 * s + 2 * h + c;  // 16 of K
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              uint32_t y[kParts<T>][2];
              if constexpr (kWhole) {
                operand_pairs(x.v[j][in], y);
              } else {
                T v[4];
                const int b = warp + i * kWarps, k = b * kBlockK + 16 * in;
                if (b < whole_blocks)
                  load4(row[j] + k, 4, true, v);
                else
                  load4(row[j] + k, a.K - (k + 4 * t), a.wide_x, v);
                operand_pairs(v, y);
              }
#pragma unroll
              for (int f = 0; f < kParts<T>; ++f) mma_w4<T>(d[j], p[2 * c], q[2 * c], p[2 * c + 1], q[2 * c + 1], y[f][0], y[f][1]);
            }
          }
          if (h == 0 && group_shift == 5) {
            scaled(2 * s);
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) d[j][e] = 0.0f;
          }
        }
        // (groups of 32: the second of these 64)
        scaled((s == 1 ? second_group : 0u) + (group_shift == 5 ? 1u : 0u));
      }
    }
  };
  if constexpr (kAhead) {
    Tokens x[2];
    if (mine > 0) load_tokens(0, x[0]);
    for (int i = 0; i < mine; i += kRing)
#pragma unroll
      for (int u = 0; u < kRing; ++u) {
        if (i + u >= mine) break;
        if (i + u + 1 < mine) load_tokens(i + u + 1, x[(u + 1) & 1]);
        multiply(i + u, u, x[u & 1]);
      }
  } else {
    Tokens x;
    for (int i = 0; i < mine; i += kRing)
#pragma unroll
      for (int u = 0; u < kRing; ++u) {
        if (i + u >= mine) break;
        if constexpr (kWhole) load_tokens(i + u, x);
        multiply(i + u, u, x);
      }
  }
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[warp][n * NT + j][2 * t + (e & 1)][g + 8 * (e >> 1)] = sum[n][j][e];
  __syncthreads();
  for (int e = threadIdx.x; e < NS * NT * 128; e += 32 * kWarps) {
    const int r = e & 15, c = (e >> 4) & 7, j = e >> 7;
    const int n = (strip + j / NT) * 16 + r;
    const int64_t m = m0 + 8 * (j % NT) + c;
    if (n >= a.N || m >= a.M) continue;
    float y = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) y += part[w][j][c][r];
    put_w4(a, m, n, a.bias != nullptr ? y + a.bias[n] : y);
  }
}

template <typename T, typename S, int NT, int NS, int kRing>
cudaError_t launch_rows_as(const W4Args& a, cudaStream_t s) {
  constexpr int kSmem = kWarps * kRing * NS * kPlace;
  static int attr_set[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(pq_linear_w4_rows<T, S, NT, NS, kRing>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    if (dev < 64) attr_set[dev] = 1;
  }
  const dim3 grid(static_cast<unsigned>((a.p.strips + NS - 1) / NS), static_cast<unsigned>((a.M + 8 * NT - 1) / (8 * NT)));
  pq_linear_w4_rows<T, S, NT, NS, kRing><<<grid, 32 * kWarps, kSmem, s>>>(a);
  return cudaGetLastError();
}

template <typename T, typename S>
cudaError_t launch_rows(const W4Args& a, cudaStream_t s) {
  // Two strips a block where the chip is full all the same, for the tokens' sake (us, two strips against one: 8 x 16384 x 8192 22.2 /
  // 28.4, one token 19.7 / 19.3; 16 x 4096 x 4096 7.4 / 8.2, 16 x 8192 x 4096 10.7 / 19.0; one x 4096 x 4096 5.3 / 5.0).
  if (a.M <= 8) return a.p.strips >= 608 ? launch_rows_as<T, S, 1, 2, 2>(a, s) : launch_rows_as<T, S, 1, 1, 4>(a, s);
  if (a.M <= 16) return a.p.strips >= 128 ? launch_rows_as<T, S, 2, 2, 2>(a, s) : launch_rows_as<T, S, 2, 1, 4>(a, s);
  return launch_rows_as<T, S, 4, 1, 4>(a, s);
}

}  // namespace

template <typename T>
cudaError_t launch_w4_rows(const W4Args& a, cudaStream_t s) {
  return a.p.s_type == PQ_F32 ? launch_rows<T, float>(a, s) : a.p.s_type == PQ_F16 ? launch_rows<T, __half>(a, s) : launch_rows<T, __nv_bfloat16>(a, s);
}

}  // namespace pq
