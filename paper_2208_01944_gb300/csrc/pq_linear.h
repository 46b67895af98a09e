// What the dense-layer kernels on 8-bit codes share.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "palquant.h"
#include "pq_tokens.cuh"

namespace pq {

struct LinearArgs {
  const void* q;
  int64_t ldq;
  const float* s_x;
  const int8_t* w;
  int64_t ldw;
  const float* s_w;
  const float* bias;
  int32_t* acc;
  void* y;
  int64_t ldy;
  int64_t M;
  int N, K;
  int y_type;
  bool wide_q;  // token rows on 16-byte boundaries
};

struct LinearTc {
  LinearArgs a;
  int n_tiles, m_tiles;  // tiles of 128 channels, of BN tokens
  int k_parts;           // blocks of a cluster that share a tile's K (1: none)
  unsigned int* err;
  uint64_t wait_limit_ns;
};

// One output: s_x is token m's, s_w and bias are channel n's.
__device__ __forceinline__ void put_result(const LinearArgs& a, int64_t m, int n, int acc, float s_x, float s_w, float bias) {
  if (a.acc != nullptr) a.acc[m * a.N + n] = acc;
  if (a.y == nullptr) return;
  float y = __fmul_rn(__fmul_rn(__int2float_rn(acc), s_x), s_w);
  if (a.bias != nullptr) y = __fadd_rn(y, bias);
  const int64_t at = m * a.ldy + n;
  if (a.y_type == PQ_F32)
    static_cast<float*>(a.y)[at] = y;
  else if (a.y_type == PQ_F16)
    static_cast<__half*>(a.y)[at] = __float2half_rn(y);
  else
    static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(y);
}

// The tensor-core kernel takes half codes in 16-byte aligned rows.
bool linear_tc_takes(const LinearArgs& a);
cudaError_t launch_linear_tc(const LinearArgs& a, bool after_tokens, cudaStream_t stream);

// Tensor map of a matrix with `cols` contiguous elements a row; out-of-range elements are zero.
bool encode_map_2d(CUtensorMap* map, CUtensorMapDataType type, const void* base, uint64_t cols, uint64_t rows,
                   uint64_t pitch_bytes, uint32_t box_cols, uint32_t box_rows, CUtensorMapSwizzle swizzle);

}  // namespace pq
