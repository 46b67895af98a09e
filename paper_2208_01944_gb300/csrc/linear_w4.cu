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
#include "pq_w4.cuh"

namespace pq {
namespace {

constexpr int kWarps = 8;

__device__ __forceinline__ void store_scale(void* at, int type, float s) {
  if (type == PQ_F32)
    *static_cast<float*>(at) = s;
  else if (type == PQ_F16)
    *static_cast<__half*>(at) = __float2half_rn(s);
  else
    *static_cast<__nv_bfloat16*>(at) = __float2bfloat16_rn(s);
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

// ------------------------------------------------------------------- packing
// A thread a word (8 codes of a row), row by row; the first word's thread of a group takes its scale along.
__global__ void __launch_bounds__(256) pq_w4_pack(const int8_t* __restrict__ codes, int64_t ldc, const uint8_t* __restrict__ scales,
                                                  PackedW4 p, int N, int K, uint8_t* __restrict__ out) {
  const int64_t words = static_cast<int64_t>(p.blocks) * (kBlockK / 8), total = words * p.strips * 16;
  const int groups = (K + (1 << p.group_shift) - 1) >> p.group_shift;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t n = i / words;
    const int at = static_cast<int>(i - n * words), r = static_cast<int>(n & 15);
    uint8_t* strip = out + (n >> 4) * p.strip_bytes();
    uint32_t word = 0;
    if (n < N)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (column_of(at, j) < K) word |= static_cast<uint32_t>(codes[n * ldc + column_of(at, j)] & 15) << nibble_shift(j);
    *reinterpret_cast<uint32_t*>(strip + word_at(p, r, at)) = word;
    if ((at * 8 & ((1 << p.group_shift) - 1)) == 0) {
      const int g = at * 8 >> p.group_shift;
      const bool there = n < N && g < groups;
      uint8_t* to = strip + scale_at(p, r, g);
      for (int b = 0; b < p.s_bytes; ++b) to[b] = there ? scales[(n * groups + g) * p.s_bytes + b] : 0;
    }
  }
}

__global__ void __launch_bounds__(256) pq_w4_unpack(const uint8_t* __restrict__ packed, PackedW4 p, int N, int K,
                                                    int8_t* __restrict__ codes, int64_t ldc, float* __restrict__ scales) {
  const int64_t words = (K + 31) / 32 * 4, total = words * N;
  const int groups = (K + (1 << p.group_shift) - 1) >> p.group_shift;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t n = i / words;
    const int at = static_cast<int>(i - n * words), r = static_cast<int>(n & 15);
    const uint8_t* strip = packed + (n >> 4) * p.strip_bytes();
    const uint32_t word = *reinterpret_cast<const uint32_t*>(strip + word_at(p, r, at));
    if (codes != nullptr)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (column_of(at, j) < K)
          codes[n * ldc + column_of(at, j)] = static_cast<int8_t>(static_cast<int>((word >> nibble_shift(j) & 15u) ^ 8u) - 8);
    if (scales != nullptr && (at * 8 & ((1 << p.group_shift) - 1)) == 0) {
      const int g = at * 8 >> p.group_shift;
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
    const int at = static_cast<int>(i - n * words), r = static_cast<int>(n & 15);
    Vec8<T> v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = column_of(at, 4 * h);
      T part[4];
      load4(x + (n < N ? n * ldx + min(k, K - 1) : 0), n < N ? K - k : 0, wide, part);
#pragma unroll
      for (int j = 0; j < 4; ++j) v.v[4 * h + j] = part[j];
    }
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
    *reinterpret_cast<uint32_t*>(strip + word_at(p, r, at)) = word;
    if ((at * 8 & ((1 << p.group_shift) - 1)) == 0) store_scale(strip + scale_at(p, r, at * 8 >> p.group_shift), p.s_type, scale);
  }
}

// ------------------------------------------------------------------ products
// Rows g's and g + 8's scale of a group, neighbours in shared memory.
__device__ __forceinline__ void scale_pair(uint32_t at, int type, float& s0, float& s1) {
  if (type == PQ_F32) {
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(s0), "=f"(s1) : "r"(at) : "memory");
    return;
  }
  uint32_t w;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
  if (type == PQ_F16) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    s0 = f.x, s1 = f.y;
  } else {
    s0 = __uint_as_float(w << 16), s1 = __uint_as_float(w & 0xFFFF0000u);
  }
}

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

// A block: 16 channels x 8 NT tokens; its warps take the strip's blocks of 128 of K in turn.  The weights come through
// rings of asynchronous copies, one for each warp (a block of 128 of K a stage, RING - 1 of them ahead, so that 32 warps keep
// 100 KB in flight on an SM); each lane reads codes that it copied itself, and scales that its warp copied.  The tokens,
// which every block reads, come from L1 and L2 into registers, a block of K ahead where they fit.
constexpr int kMostBlock = 1024 + 256;  // bytes of 128 of K of a strip: four groups' fp32 scales

template <typename T, int NT, int RING>
__global__ void __launch_bounds__(32 * kWarps) pq_linear_w4_rows(const __grid_constant__ W4Args a) {
  extern __shared__ __align__(16) uint8_t ring_raw[];
  __shared__ float part[kWarps][NT][8][17];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * (8 * NT);
  const uint8_t* strip = a.w + static_cast<int64_t>(blockIdx.x) * a.p.strip_bytes();
  const uint32_t ring = smem_u32(ring_raw) + warp * RING * a.p.block_bytes;
  const int scale_pieces = (a.p.block_bytes - 1024) >> 4;
  const int mine = a.p.blocks > warp ? (a.p.blocks - warp - 1) / kWarps + 1 : 0;
  auto fetch = [&](int i, int stage) {
    const uint8_t* from = strip + static_cast<int64_t>(warp + i * kWarps) * a.p.block_bytes + lane * 16;
    const uint32_t to = ring + stage * a.p.block_bytes + lane * 16;
    cp_async_16(to, from, 16);
    cp_async_16(to + 512, from + 512, 16);
    if (lane < scale_pieces) cp_async_16(to + 1024, from + 1024, 16);
  };
#pragma unroll
  for (int i = 0; i < RING - 1; ++i) {
    if (i < mine) fetch(i, i);
    cp_async_commit();
  }
  const T* row[NT];
  bool there[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int64_t m = m0 + 8 * j + g;
    there[j] = m < a.M;
    row[j] = static_cast<const T*>(a.x) + (there[j] ? m : 0) * a.ldx;
  }
  // 16 of K of a token: columns 128 b + 16 c + 4 t and up
  auto tokens_at = [&](int j, int b, int c, T (&v)[4]) {
    const int k = b * kBlockK + 16 * c + 4 * t;
    load4(row[j] + min(k, a.K - 1), there[j] ? a.K - k : 0, a.wide_x, v);
  };
  constexpr bool kAhead = NT == 1 && sizeof(T) == 2;
  T next[kAhead ? 8 : 1][4];
  auto tokens_ahead = [&](int i) {
    if constexpr (kAhead) {
      if (i >= mine) return;
#pragma unroll
      for (int c = 0; c < 8; ++c) tokens_at(0, warp + i * kWarps, c, next[c]);
    }
  };
  tokens_ahead(0);
  float sum[NT][4] = {};
  int stage = 0;
  for (int i = 0; i < mine; ++i) {
    T now[kAhead ? 8 : 1][4];
    if constexpr (kAhead) {
#pragma unroll
      for (int c = 0; c < 8; ++c) memcpy(now[c], next[c], sizeof(now[c]));
      tokens_ahead(i + 1);
    }
    cp_async_wait<RING - 2>();
    __syncwarp();  // the block's scales have arrived, and every lane is done with the stage before
    const uint32_t at = ring + stage * a.p.block_bytes;
    {
      const int before = stage == 0 ? RING - 1 : stage - 1;
      if (i + RING - 1 < mine) fetch(i + RING - 1, before);
      cp_async_commit();
      stage = stage + 1 == RING ? 0 : stage + 1;
    }
    float d[NT][4] = {};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      uint4 u;
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                   : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w)
                   : "r"(at + s * 512 + lane * 16)
                   : "memory");
      const uint32_t words[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t p[4], q[4];
        p[0] = code_pair<T, 0>(words[2 * h]), p[1] = code_pair<T, 1>(words[2 * h]);
        p[2] = code_pair<T, 2>(words[2 * h]), p[3] = code_pair<T, 3>(words[2 * h]);
        q[0] = code_pair<T, 0>(words[2 * h + 1]), q[1] = code_pair<T, 1>(words[2 * h + 1]);
        q[2] = code_pair<T, 2>(words[2 * h + 1]), q[3] = code_pair<T, 3>(words[2 * h + 1]);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int in = 4 * s + 2 * h + c;  // 16 of K
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            uint32_t x[kParts<T>][2];
            if constexpr (kAhead) {
              operand_pairs(now[in], x);
            } else {
              T v[4];
              tokens_at(j, warp + i * kWarps, in, v);
              operand_pairs(v, x);
            }
#pragma unroll
            for (int f = 0; f < kParts<T>; ++f) mma_w4<T>(d[j], p[2 * c], q[2 * c], p[2 * c + 1], q[2 * c + 1], x[f][0], x[f][1]);
          }
        }
        // a group is over
        const int end = 64 * s + 32 * h + 32;
        if ((end & ((1 << a.p.group_shift) - 1)) == 0) {
          const int group = (end - 32) >> a.p.group_shift;
          float s0, s1;
          scale_pair(at + 1024 + (group * 16 + g * 2) * a.p.s_bytes, a.p.s_type, s0, s1);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            sum[j][0] = fmaf(s0, d[j][0], sum[j][0]);
            sum[j][1] = fmaf(s0, d[j][1], sum[j][1]);
            sum[j][2] = fmaf(s1, d[j][2], sum[j][2]);
            sum[j][3] = fmaf(s1, d[j][3], sum[j][3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) d[j][e] = 0.0f;
          }
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
    put_w4(a, m, n, a.bias != nullptr ? y + a.bias[n] : y);
  }
}

template <typename T, int NT, int RING>
cudaError_t launch_rows_as(const W4Args& a, cudaStream_t s) {
  static int attr_set[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(pq_linear_w4_rows<T, NT, RING>, cudaFuncAttributeMaxDynamicSharedMemorySize, kWarps * RING * kMostBlock);
    if (e != cudaSuccess) return e;
    if (dev < 64) attr_set[dev] = 1;
  }
  const dim3 grid(static_cast<unsigned>(a.p.strips), static_cast<unsigned>((a.M + 8 * NT - 1) / (8 * NT)));
  pq_linear_w4_rows<T, NT, RING><<<grid, 32 * kWarps, kWarps * RING * a.p.block_bytes, s>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_w4(const W4Args& a, cudaStream_t s) {
  if (a.M <= 8) return launch_rows_as<T, 1, 4>(a, s);
  if (a.M <= 16) return launch_rows_as<T, 2, 4>(a, s);
  if (a.M <= 32) return launch_rows_as<T, 4, 4>(a, s);
  return launch_rows_as<T, 8, 4>(a, s);
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
  const bool wide = pq::is_aligned(w_dev, 4 * pq::bytes_of_type(w_type)) && ldw % 4 == 0;
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
                        d->N, d->K, d->y_type, pq::is_aligned(x_dev, 4 * e) && d->ldx % 4 == 0};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t st = pq::w4_tc_takes(a, d->x_type) ? pq::launch_w4_tc(a, d->x_type, s)
                         : d->x_type == PQ_F32   ? pq::launch_w4<float>(a, s)
                         : d->x_type == PQ_F16 ? pq::launch_w4<__half>(a, s)
                                               : pq::launch_w4<__nv_bfloat16>(a, s);
  return st == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

}  // extern "C"
