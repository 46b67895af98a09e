// Packed 4-bit weights, and what the dense-layer kernels on them share.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "palquant.h"
#include "pq_tokens.cuh"

namespace pq {

constexpr int kBlockK = 128;     // of K between a strip's scales
constexpr int kTileStrips = 8;

// A strip is 16 channels; eight of them (the last ones fewer) are a tile.  A tile holds, for each 128 of K, a block of every
// strip: 1024 bytes of codes (two steps of 64), then the scales of its groups.  So a tile's 128 of K are one run of bytes
// (eight copies of a strip's block each took the copying warp 1000 cycles, of the 1700 that such a stage took).  Of a step,
// lane 4 g + t holds 16 bytes: of rows g and g + 8, for each 32 of K a word of 8 codes: columns 4 t to 4 t + 3 and
// 16 + 4 t to 16 + 4 t + 3.  That is an operand of two 16 x 16 MMAs, and in tensor memory a row's 64-bit piece.
struct PackedW4 {
  int strips, blocks;  // of 128 of K
  int group_shift;     // log2(group): 5 to 7
  int s_type, s_bytes;
  int block_bytes;
  // strips of a tile, where a strip begins, and the bytes from one of its blocks to the next
  __host__ __device__ int strips_of(int tile) const { return strips - tile * kTileStrips < kTileStrips ? strips - tile * kTileStrips : kTileStrips; }
  __host__ __device__ int64_t strip_at(int strip) const {
    const int tile = strip / kTileStrips;
    return (static_cast<int64_t>(tile) * kTileStrips * blocks + strip % kTileStrips) * block_bytes;
  }
  __host__ __device__ int pitch(int strip) const { return strips_of(strip / kTileStrips) * block_bytes; }
};

inline PackedW4 packed_of(const pq_w4_weights* w) {
  PackedW4 p;
  p.strips = (w->N + 15) / 16;
  p.blocks = (w->K + kBlockK - 1) / kBlockK;
  p.group_shift = w->group == 32 ? 5 : w->group == 64 ? 6 : 7;
  p.s_type = w->s_type;
  p.s_bytes = static_cast<int>(bytes_of_type(w->s_type));
  p.block_bytes = 1024 + (kBlockK >> p.group_shift) * 16 * p.s_bytes;
  return p;
}

// Where word i of channel n (words 4 b to 4 b + 3 hold columns 32 b to 32 b + 31) lies, and channel n's scale of group g.
__host__ __device__ inline int64_t word_at(const PackedW4& p, int n, int i) {
  const int r = n & 15, in = i & 15, step = in >> 3, half = (in >> 2) & 1, t = in & 3;
  return p.strip_at(n >> 4) + static_cast<int64_t>(i >> 4) * p.pitch(n >> 4) + step * 512 + ((r & 7) * 4 + t) * 16 + half * 8 + (r >> 3) * 4;
}
// Column of code j of word i, and its place in the word: pairs (j, j + 1) lie 16 bits apart.
__host__ __device__ constexpr int column_of(int i, int j) { return 32 * (i >> 2) + 4 * (i & 3) + (j & 3) + 16 * (j >> 2); }
__host__ __device__ inline int64_t scale_at(const PackedW4& p, int n, int g) {
  const int r = n & 15, per = kBlockK >> p.group_shift;
  return p.strip_at(n >> 4) + static_cast<int64_t>(g / per) * p.pitch(n >> 4) + 1024 + ((g % per) * 16 + (r & 7) * 2 + (r >> 3)) * p.s_bytes;
}
__host__ __device__ constexpr int nibble_shift(int j) { return 4 * ((j & 1) * 4 + (j >> 1)); }

__device__ __forceinline__ float load_scale(const void* at, int type) {
  if (type == PQ_F32) return *static_cast<const float*>(at);
  if (type == PQ_F16) return __half2float(*static_cast<const __half*>(at));
  return __bfloat162float(*static_cast<const __nv_bfloat16*>(at));
}

struct W4Args {
  PackedW4 p;
  const void* x;
  const uint8_t* w;
  const float* bias;
  void* y;
  int64_t ldx, ldy, M;
  int N, K, y_type;
  bool wide_x;  // four elements of a token row lie on a boundary of their size
};

// Few tokens, and any alignment and type: 8 to 32 tokens a tile.
template <typename T>
cudaError_t launch_w4_rows(const W4Args& a, cudaStream_t stream);

// Up to 128 tokens a tile on the tensor cores.  Scratch: a copy of tokens that it cannot load where they are (16-bit ones whose rows
// begin off 16-byte boundaries; without a pitch that shows it, the other kernel takes them).
size_t w4_tc_scratch(int64_t M, int N, int K, int64_t ldx, int x_type);
bool w4_tc_takes(const W4Args& a, int x_type);
cudaError_t launch_w4_tc(const W4Args& a, int x_type, void* scratch, cudaStream_t stream);

// One output, in fp32 until here.
__device__ __forceinline__ void put_w4(const W4Args& a, int64_t m, int n, float y) {
  const int64_t at = m * a.ldy + n;
  if (a.y_type == PQ_F32)
    static_cast<float*>(a.y)[at] = y;
  else if (a.y_type == PQ_F16)
    static_cast<__half*>(a.y)[at] = __float2half_rn(y);
  else
    static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(y);
}

// How activations enter the products: halves, bfloat16, or fp32 as three bfloat16 parts.
template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 3 : 1;

// Four activations as two pairs, part by part.
template <typename T>
__device__ __forceinline__ void operand_pairs(const T (&v)[4], uint32_t (&r)[kParts<T>][2]) {
  if constexpr (sizeof(T) == 2) {
    memcpy(r[0], v, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t part[2][3];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        // 8 + 8 + 8 bits by truncation; an infinity or a NaN is its first part alone
        const float x = v[2 * i + j];
        const uint32_t hi = __float_as_uint(x) & 0xFFFF0000u;
        const bool finite = (hi & 0x7F800000u) != 0x7F800000u;
        const float rest = finite ? x - __uint_as_float(hi) : 0.0f;
        const uint32_t mid = __float_as_uint(rest) & 0xFFFF0000u;
        part[j][0] = finite || hi == __float_as_uint(x) ? hi : hi | 0x00400000u;
        part[j][1] = mid;
        part[j][2] = __float_as_uint(rest - __uint_as_float(mid));
      }
#pragma unroll
      for (int h = 0; h < 3; ++h) r[h][i] = __byte_perm(part[0][h], part[1][h], 0x7632);
    }
  }
}

// n of four consecutive elements (the others zero); `wide`: their address is a multiple of their size.
template <typename T>
__device__ __forceinline__ void load4(const T* p, int n, bool wide, T (&v)[4]) {
  if (wide && n >= 4) {
    if constexpr (sizeof(T) == 2) {
      const uint2 q = *reinterpret_cast<const uint2*>(p);
      memcpy(v, &q, 8);
    } else {
      const uint4 q = *reinterpret_cast<const uint4*>(p);
      memcpy(v, &q, 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? p[i] : from_f32<T>(0.0f);
  }
}

// Small integers put under the exponent of a power of two and that power subtracted: a published way of converting 4-bit codes (Kim et
// al., "Who Says Elephants Can't Run", 2022, arXiv 2211.10017).  Pair i (columns 2 i and 2 i + 1) of a word's codes in the products' type: the
// code's sign bit is flipped under the
// exponent of 1024 (128): 1032 + c (136 + c).
template <typename T, int I>
__device__ __forceinline__ uint32_t code_pair(uint32_t word) {
  if constexpr (sizeof(T) == 2 && !std::is_same<T, __nv_bfloat16>::value) {
    return sub_half2(((word >> (4 * I)) & 0x000F000Fu) ^ 0x64086408u, 0x64086408u);
  } else {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(((word >> (4 * I)) & 0x000F000Fu) ^ 0x43084308u), "r"(0x43084308u));
    return r;
  }
}

// The four pairs of a word.  Halves hold 10 bits behind 1024, so a pair 4 bits up needs no shift: 1024 + 16 (8 + c), over 16.
template <typename T>
__device__ __forceinline__ void code_pairs(uint32_t word, uint32_t (&r)[4]) {
  if constexpr (sizeof(T) == 2 && !std::is_same<T, __nv_bfloat16>::value) {
    const uint32_t up = word >> 8;
    r[0] = sub_half2((word & 0x000F000Fu) ^ 0x64086408u, 0x64086408u);
    r[2] = sub_half2((up & 0x000F000Fu) ^ 0x64086408u, 0x64086408u);
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r[1]) : "r"((word & 0x00F000F0u) ^ 0x64806480u), "r"(0x2C002C00u), "r"(0xD480D480u));
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r[3]) : "r"((up & 0x00F000F0u) ^ 0x64806480u), "r"(0x2C002C00u), "r"(0xD480D480u));
  } else {
    r[0] = code_pair<T, 0>(word), r[1] = code_pair<T, 1>(word), r[2] = code_pair<T, 2>(word), r[3] = code_pair<T, 3>(word);
  }
}

}  // namespace pq
