// Dense layers with 4-bit weights and a scale for each output channel and group of input channels.
//
// Mathematics.  y[m, n] = sum_g s[n, g] sum_{k in g} c[n, k] x[m, k].  A code is an integer in [-8, 7], exact in
// half precision and in bfloat16, so 16-bit activations are multiplied as they are, and an fp32 activation is
// cut into three bfloat16 parts of 8 bits each (by truncation: exact).  Every product is exact, a group's sums are
// fp32, and its scale multiplies them in fp32.
//
// Layout.  Weights are packed once in the order in which the products take them (PackedW4): a strip of 16 output
// channels is the MMA's 16 rows, a warp's 512 bytes are 64 of K, a lane's 16 bytes are its operands of four MMAs;
// the group's scales follow every 128 of K.  Two codes lie 16 bits apart, so that one logic operation puts
// both under the exponent of 128 (bfloat16) or 1024 (half), and one subtraction leaves them: 11 instructions for 8 codes.
#include <cuda_runtime.h>

#include <algorithm>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_tokens.cuh"

namespace pq {
namespace {

constexpr int kBlockK = 128;  // of K between a strip's scales
constexpr int kWarps = 8;

// A strip of 16 channels: for each 128 of K, 1024 bytes of codes (two steps of 64), then the scales of its groups.
struct PackedW4 {
  int strips, blocks;  // of 128 of K
  int group_shift;     // log2(group): 5 to 7
  int s_type, s_bytes;
  int block_bytes;
  __host__ __device__ int64_t strip_bytes() const { return static_cast<int64_t>(blocks) * block_bytes; }
};

PackedW4 packed_of(const pq_w4_weights* w) {
  PackedW4 p;
  p.strips = (w->N + 15) / 16;
  p.blocks = (w->K + kBlockK - 1) / kBlockK;
  p.group_shift = w->group == 32 ? 5 : w->group == 64 ? 6 : 7;
  p.s_type = w->s_type;
  p.s_bytes = static_cast<int>(bytes_of_type(w->s_type));
  p.block_bytes = 1024 + (kBlockK >> p.group_shift) * 16 * p.s_bytes;
  return p;
}

// Where the word of row r's 8 codes from column k on (a multiple of 8) lies in a strip, and row r's scale of group g.
__host__ __device__ inline int64_t word_at(const PackedW4& p, int r, int k) {
  const int in = k & (kBlockK - 1), step = in >> 6, half = (in >> 5) & 1, t = (in >> 3) & 3;
  return static_cast<int64_t>(k / kBlockK) * p.block_bytes + step * 512 + ((r & 7) * 4 + t) * 16 + half * 8 + (r >> 3) * 4;
}
__host__ __device__ inline int64_t scale_at(const PackedW4& p, int r, int g) {
  const int per = kBlockK >> p.group_shift;
  return static_cast<int64_t>(g / per) * p.block_bytes + 1024 + ((g % per) * 16 + (r & 7) * 2 + (r >> 3)) * p.s_bytes;
}
// The place of column k's code in its word: pairs (k, k + 1) lie 16 bits apart.
__host__ __device__ constexpr int nibble_shift(int k) { return 4 * ((k & 1) * 4 + ((k & 7) >> 1)); }

__device__ __forceinline__ float load_scale(const void* at, int type) {
  if (type == PQ_F32) return *static_cast<const float*>(at);
  if (type == PQ_F16) return __half2float(*static_cast<const __half*>(at));
  return __bfloat162float(*static_cast<const __nv_bfloat16*>(at));
}
__device__ __forceinline__ void store_scale(void* at, int type, float s) {
  if (type == PQ_F32)
    *static_cast<float*>(at) = s;
  else if (type == PQ_F16)
    *static_cast<__half*>(at) = __float2half_rn(s);
  else
    *static_cast<__nv_bfloat16*>(at) = __float2bfloat16_rn(s);
}

// ------------------------------------------------------------------- packing
// A thread a word (8 codes of a row), row by row; the first 8 columns' threads of a group take its scale along.
__global__ void __launch_bounds__(256) pq_w4_pack(const int8_t* __restrict__ codes, int64_t ldc, const uint8_t* __restrict__ scales,
                                                  PackedW4 p, int N, int K, uint8_t* __restrict__ out) {
  const int64_t words = static_cast<int64_t>(p.blocks) * (kBlockK / 8), total = words * p.strips * 16;
  const int groups = (K + (1 << p.group_shift) - 1) >> p.group_shift;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t n = i / words;
    const int k = static_cast<int>(i - n * words) * 8, r = static_cast<int>(n & 15);
    uint8_t* strip = out + (n >> 4) * p.strip_bytes();
    uint32_t word = 0;
    if (n < N)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k + j < K) word |= static_cast<uint32_t>(codes[n * ldc + k + j] & 15) << nibble_shift(j);
    *reinterpret_cast<uint32_t*>(strip + word_at(p, r, k)) = word;
    if ((k & ((1 << p.group_shift) - 1)) == 0) {
      const int g = k >> p.group_shift;
      const bool there = n < N && g < groups;
      uint8_t* to = strip + scale_at(p, r, g);
      for (int b = 0; b < p.s_bytes; ++b) to[b] = there ? scales[(n * groups + g) * p.s_bytes + b] : 0;
    }
  }
}

__global__ void __launch_bounds__(256) pq_w4_unpack(const uint8_t* __restrict__ packed, PackedW4 p, int N, int K,
                                                    int8_t* __restrict__ codes, int64_t ldc, float* __restrict__ scales) {
  const int64_t words = (K + 7) / 8, total = words * N;
  const int groups = (K + (1 << p.group_shift) - 1) >> p.group_shift;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t n = i / words;
    const int k = static_cast<int>(i - n * words) * 8, r = static_cast<int>(n & 15);
    const uint8_t* strip = packed + (n >> 4) * p.strip_bytes();
    const uint32_t word = *reinterpret_cast<const uint32_t*>(strip + word_at(p, r, k));
    if (codes != nullptr)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k + j < K) codes[n * ldc + k + j] = static_cast<int8_t>(static_cast<int>((word >> nibble_shift(j) & 15u) ^ 8u) - 8);
    if (scales != nullptr && (k & ((1 << p.group_shift) - 1)) == 0) {
      const int g = k >> p.group_shift;
      scales[n * groups + g] = load_scale(strip + scale_at(p, r, g), p.s_type);
    }
  }
}

// Scale of a group as it is stored: amax / 7 in s_type, 0 below that type's normal numbers, NaN where it cannot be held.
__device__ __forceinline__ float w4_scale(uint32_t amax, int type) {
  if (amax >= 0x7F800000u) return __int_as_float(0x7FC00000);
  float s = __fmul_rn(__uint_as_float(amax), 1.0f / 7.0f);
  if (type == PQ_F16) s = __half2float(__float2half_rn(s));
  if (type == PQ_BF16) s = __bfloat162float(__float2bfloat16_rn(s));
  if (s < (type == PQ_F16 ? 0x1p-14f : FLT_MIN)) return 0.0f;
  return s <= FLT_MAX ? s : __int_as_float(0x7FC00000);
}

// A thread a word; the threads of a group are neighbours (4, 8 or 16 of them) and share its largest magnitude.
template <typename T>
__global__ void __launch_bounds__(256) pq_w4_quantize(const T* __restrict__ x, int64_t ldx, PackedW4 p, int N, int K,
                                                      uint8_t* __restrict__ out, bool wide) {
  const int64_t words = static_cast<int64_t>(p.blocks) * (kBlockK / 8), total = words * p.strips * 16;  // a multiple of 256
  const int members = 1 << (p.group_shift - 3);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t n = i / words;
    const int k = static_cast<int>(i - n * words) * 8, r = static_cast<int>(n & 15);
    const int left = n < N ? K - k : 0;
    const Vec8<T> v = load8(x + (n < N ? n * ldx + min(k, K - 1) : 0), left, wide && left >= 8);
    uint32_t top = amax8(v);
    for (int s = 1; s < members; s <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
    const float scale = w4_scale(top, p.s_type), inv = inverse_of_scale(scale);
    uint32_t word = 0;
    if (inv > 0.0f)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = min(7, max(-7, __float2int_rn(__fmul_rn(to_f32(v.v[j]), inv))));
        word |= static_cast<uint32_t>(c & 15) << nibble_shift(j);
      }
    uint8_t* strip = out + (n >> 4) * p.strip_bytes();
    *reinterpret_cast<uint32_t*>(strip + word_at(p, r, k)) = word;
    if ((k & ((1 << p.group_shift) - 1)) == 0) store_scale(strip + scale_at(p, r, k >> p.group_shift), p.s_type, scale);
  }
}

// ------------------------------------------------------------------ products
struct W4Args {
  PackedW4 p;
  const void* x;
  const uint8_t* w;
  const float* bias;
  void* y;
  int64_t ldx, ldy, M;
  int N, K, y_type;
  bool wide_x;  // token rows on 16-byte boundaries
};

// How activations enter the products: halves, bfloat16, or fp32 as three bfloat16 parts.
template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 3 : 1;

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

// Pair i (columns 2 i and 2 i + 1) of a word's codes in the products' type.  The code's sign bit is flipped under the
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

// Eight activations as pairs, part by part.
template <typename T>
__device__ __forceinline__ void operand_pairs(const Vec8<T>& v, uint32_t (&r)[kParts<T>][4]) {
  if constexpr (sizeof(T) == 2) {
    memcpy(r[0], &v, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t part[2][3];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        // 8 + 8 + 8 bits by truncation; an infinity or a NaN is its first part alone
        const float x = to_f32(v.v[2 * i + j]);
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

// A block: 16 channels x 8 NT tokens; its warps take the strip's blocks of 128 of K in turn.
template <typename T, int NT>
__global__ void __launch_bounds__(32 * kWarps) pq_linear_w4_rows(const __grid_constant__ W4Args a) {
  __shared__ float part[kWarps][NT][8][17];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * (8 * NT);
  const uint8_t* strip = a.w + static_cast<int64_t>(blockIdx.x) * a.p.strip_bytes();
  const T* row[NT];
  bool there[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t m = m0 + 8 * j + g;
    there[j] = m < a.M;
    row[j] = static_cast<const T*>(a.x) + (there[j] ? m : 0) * a.ldx;
  }
  float sum[NT][4] = {};
  for (int b = warp; b < a.p.blocks; b += kWarps) {
    const uint8_t* block = strip + static_cast<int64_t>(b) * a.p.block_bytes;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint4 u = *reinterpret_cast<const uint4*>(block + s * 512 + lane * 16);
      const uint32_t words[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int in = 64 * s + 32 * h, k = b * kBlockK + in + 8 * t;
        const uint8_t* at = block + 1024 + ((in >> a.p.group_shift) * 16 + g * 2) * a.p.s_bytes;
        const float s0 = load_scale(at, a.p.s_type), s1 = load_scale(at + a.p.s_bytes, a.p.s_type);
        const uint32_t p0 = code_pair<T, 0>(words[2 * h]), p1 = code_pair<T, 1>(words[2 * h]),
                       p2 = code_pair<T, 2>(words[2 * h]), p3 = code_pair<T, 3>(words[2 * h]);
        const uint32_t q0 = code_pair<T, 0>(words[2 * h + 1]), q1 = code_pair<T, 1>(words[2 * h + 1]),
                       q2 = code_pair<T, 2>(words[2 * h + 1]), q3 = code_pair<T, 3>(words[2 * h + 1]);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int left = there[j] ? a.K - k : 0;
          const Vec8<T> v = load8(row[j] + min(k, a.K - 1), left, a.wide_x && left >= 8);
          uint32_t x[kParts<T>][4];
          operand_pairs(v, x);
          float d[4] = {};
#pragma unroll
          for (int i = 0; i < kParts<T>; ++i) {
            mma_w4<T>(d, p0, q0, p1, q1, x[i][0], x[i][1]);
            mma_w4<T>(d, p2, q2, p3, q3, x[i][2], x[i][3]);
          }
          sum[j][0] = fmaf(s0, d[0], sum[j][0]);
          sum[j][1] = fmaf(s0, d[1], sum[j][1]);
          sum[j][2] = fmaf(s1, d[2], sum[j][2]);
          sum[j][3] = fmaf(s1, d[3], sum[j][3]);
        }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[warp][j][2 * t + (e & 1)][g + 8 * (e >> 1)] = sum[j][e];
  __syncthreads();
  for (int e = threadIdx.x; e < NT * 128; e += 32 * kWarps) {
    const int r = e & 15, c = (e >> 4) & 7, j = e >> 7;
    const int n = blockIdx.x * 16 + r;
    const int64_t m = m0 + 8 * j + c;
    if (n >= a.N || m >= a.M) continue;
    float y = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) y += part[w][j][c][r];
    if (a.bias != nullptr) y += a.bias[n];
    const int64_t at = m * a.ldy + n;
    if (a.y_type == PQ_F32)
      static_cast<float*>(a.y)[at] = y;
    else if (a.y_type == PQ_F16)
      static_cast<__half*>(a.y)[at] = __float2half_rn(y);
    else
      static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(y);
  }
}

template <typename T, int NT>
cudaError_t launch_rows_as(const W4Args& a, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.p.strips), static_cast<unsigned>((a.M + 8 * NT - 1) / (8 * NT)));
  pq_linear_w4_rows<T, NT><<<grid, 32 * kWarps, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_w4(const W4Args& a, cudaStream_t s) {
  if (a.M <= 8) return launch_rows_as<T, 1>(a, s);
  if (a.M <= 16) return launch_rows_as<T, 2>(a, s);
  if (a.M <= 32) return launch_rows_as<T, 4>(a, s);
  return launch_rows_as<T, 8>(a, s);
}

bool valid_w4_type(int32_t t) { return t == PQ_F32 || t == PQ_F16 || t == PQ_BF16; }

bool valid_w4(const pq_w4_weights* w) {
  return w != nullptr && w->N >= 1 && w->K >= 1 && w->K <= 131072 && w->N <= 0x7FFFFFF0 &&
         (w->group == 32 || w->group == 64 || w->group == 128) && valid_w4_type(w->s_type);
}

bool valid_w4_call(const pq_w4_weights* w, const pq_linear_desc* d) {
  return valid_w4(w) && d != nullptr && d->M >= 0 && d->N == w->N && d->K == w->K && valid_w4_type(d->x_type) &&
         valid_w4_type(d->y_type) && d->ldx >= d->K && d->ldy >= d->N;
}

// Blocks of 256 threads for a loop over `items` of them.
unsigned loop_grid(int64_t items) { return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>((items + 255) / 256, 152 * 16))); }

int64_t words_of(const PackedW4& p) { return static_cast<int64_t>(p.strips) * 16 * p.blocks * (kBlockK / 8); }

}  // namespace
}  // namespace pq

extern "C" {

size_t palquant_w4_packed_bytes(const pq_w4_weights* w) {
  if (!pq::valid_w4(w)) return 0;
  const pq::PackedW4 p = pq::packed_of(w);
  return static_cast<size_t>(p.strips) * static_cast<size_t>(p.strip_bytes());
}

pq_status palquant_w4_pack(const int8_t* codes_dev, int64_t ldc, const void* s_dev, const pq_w4_weights* w,
                           void* packed_dev, size_t packed_bytes, pq_stream_t stream) {
  if (!pq::valid_w4(w) || codes_dev == nullptr || s_dev == nullptr || packed_dev == nullptr || ldc < w->K ||
      !pq::is_aligned(packed_dev, 16) || !pq::is_aligned(s_dev, pq::bytes_of_type(w->s_type)) ||
      packed_bytes < palquant_w4_packed_bytes(w))
    return PQ_EINVAL;
  const pq::PackedW4 p = pq::packed_of(w);
  pq::pq_w4_pack<<<pq::loop_grid(pq::words_of(p)), 256, 0, static_cast<cudaStream_t>(stream)>>>(
      codes_dev, ldc, static_cast<const uint8_t*>(s_dev), p, w->N, w->K, static_cast<uint8_t*>(packed_dev));
  return cudaGetLastError() == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

pq_status palquant_w4_quantize(const void* w_dev, int32_t w_type, int64_t ldw, const pq_w4_weights* w,
                               void* packed_dev, size_t packed_bytes, pq_stream_t stream) {
  if (!pq::valid_w4(w) || !pq::valid_w4_type(w_type) || w_dev == nullptr || packed_dev == nullptr || ldw < w->K ||
      !pq::is_aligned(packed_dev, 16) || !pq::is_aligned(w_dev, pq::bytes_of_type(w_type)) ||
      packed_bytes < palquant_w4_packed_bytes(w))
    return PQ_EINVAL;
  const pq::PackedW4 p = pq::packed_of(w);
  const bool wide = pq::is_aligned(w_dev, 16) && ldw * pq::bytes_of_type(w_type) % 16 == 0;
  const unsigned grid = pq::loop_grid(pq::words_of(p));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  uint8_t* out = static_cast<uint8_t*>(packed_dev);
  if (w_type == PQ_F32)
    pq::pq_w4_quantize<float><<<grid, 256, 0, s>>>(static_cast<const float*>(w_dev), ldw, p, w->N, w->K, out, wide);
  else if (w_type == PQ_F16)
    pq::pq_w4_quantize<__half><<<grid, 256, 0, s>>>(static_cast<const __half*>(w_dev), ldw, p, w->N, w->K, out, wide);
  else
    pq::pq_w4_quantize<__nv_bfloat16><<<grid, 256, 0, s>>>(static_cast<const __nv_bfloat16*>(w_dev), ldw, p, w->N, w->K, out, wide);
  return cudaGetLastError() == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

pq_status palquant_w4_unpack(const void* packed_dev, const pq_w4_weights* w, int8_t* codes_dev, int64_t ldc,
                             float* s_dev, pq_stream_t stream) {
  if (!pq::valid_w4(w) || packed_dev == nullptr || (codes_dev == nullptr && s_dev == nullptr) ||
      (codes_dev != nullptr && ldc < w->K) || !pq::is_aligned(packed_dev, 16) || !pq::is_aligned(s_dev, 4))
    return PQ_EINVAL;
  const pq::PackedW4 p = pq::packed_of(w);
  pq::pq_w4_unpack<<<pq::loop_grid(static_cast<int64_t>(w->N) * ((w->K + 7) / 8)), 256, 0, static_cast<cudaStream_t>(stream)>>>(
      static_cast<const uint8_t*>(packed_dev), p, w->N, w->K, codes_dev, ldc, s_dev);
  return cudaGetLastError() == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

size_t palquant_linear_w4_scratch_bytes(const pq_w4_weights* w, const pq_linear_desc* d) {
  if (!pq::valid_w4_call(w, d)) return 0;
  return 0;
}

pq_status palquant_linear_w4(const void* x_dev, const void* packed_dev, const float* bias_dev, void* y_dev,
                             const pq_w4_weights* w, const pq_linear_desc* d, void* scratch_dev, size_t scratch_bytes,
                             pq_stream_t stream) {
  (void)scratch_dev;
  (void)scratch_bytes;
  if (!pq::valid_w4_call(w, d)) return PQ_EINVAL;
  if (d->M == 0) return PQ_OK;
  const size_t e = pq::bytes_of_type(d->x_type);
  if (x_dev == nullptr || packed_dev == nullptr || y_dev == nullptr || !pq::is_aligned(x_dev, e) ||
      !pq::is_aligned(packed_dev, 16) || !pq::is_aligned(bias_dev, 4) || !pq::is_aligned(y_dev, pq::bytes_of_type(d->y_type)))
    return PQ_EINVAL;
  if (d->M > 64ll * 65535) return PQ_EUNSUPPORTED;  // blocks along the grid's second axis
  const pq::W4Args a = {pq::packed_of(w), x_dev, static_cast<const uint8_t*>(packed_dev), bias_dev, y_dev, d->ldx, d->ldy, d->M,
                        d->N, d->K, d->y_type, pq::is_aligned(x_dev, 16) && d->ldx * e % 16 == 0};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t st = d->x_type == PQ_F32   ? pq::launch_w4<float>(a, s)
                         : d->x_type == PQ_F16 ? pq::launch_w4<__half>(a, s)
                                               : pq::launch_w4<__nv_bfloat16>(a, s);
  return st == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

}  // extern "C"
