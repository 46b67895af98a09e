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

__device__ __forceinline__ void store_scale(void* at, int type, float s) {
  if (type == PQ_F32)
    *static_cast<float*>(at) = s;
  else if (type == PQ_F16)
    *static_cast<__half*>(at) = __float2half_rn(s);
  else
    *static_cast<__nv_bfloat16*>(at) = __float2bfloat16_rn(s);
}

// ------------------------------------------------------------------- packing
// A thread a word (8 codes of a row), row by row; the first word's thread of a group takes its scale along.  Once in a layer's life (16384 x 8192,
// groups of 128: packed from codes 129 us, from bfloat16 weights 168, unpacked 122; their bytes 30, 50 and 30).
__global__ void __launch_bounds__(256) pq_w4_pack(const int8_t* __restrict__ codes, int64_t ldc, const uint8_t* __restrict__ scales,
                                                  PackedW4 p, int N, int K, uint8_t* __restrict__ out) {
  const int64_t words = static_cast<int64_t>(p.blocks) * (kBlockK / 8), total = words * p.strips * 16;
  const int groups = (K + (1 << p.group_shift) - 1) >> p.group_shift;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t n = i / words;
    const int at = static_cast<int>(i - n * words), row = static_cast<int>(n);
    uint32_t word = 0;
    if (n < N)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (column_of(at, j) < K) word |= static_cast<uint32_t>(codes[n * ldc + column_of(at, j)] & 15) << nibble_shift(j);
    *reinterpret_cast<uint32_t*>(out + word_at(p, row, at)) = word;
    if ((at * 8 & ((1 << p.group_shift) - 1)) == 0) {
      const int g = at * 8 >> p.group_shift;
      const bool there = n < N && g < groups;
      uint8_t* to = out + scale_at(p, row, g);
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
    const int at = static_cast<int>(i - n * words), row = static_cast<int>(n);
    const uint32_t word = *reinterpret_cast<const uint32_t*>(packed + word_at(p, row, at));
    if (codes != nullptr)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (column_of(at, j) < K)
          codes[n * ldc + column_of(at, j)] = static_cast<int8_t>(static_cast<int>((word >> nibble_shift(j) & 15u) ^ 8u) - 8);
    if (scales != nullptr && (at * 8 & ((1 << p.group_shift) - 1)) == 0) {
      const int g = at * 8 >> p.group_shift;
      scales[n * groups + g] = load_scale(packed + scale_at(p, row, g), p.s_type);
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
    const int at = static_cast<int>(i - n * words), row = static_cast<int>(n);
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
    *reinterpret_cast<uint32_t*>(out + word_at(p, row, at)) = word;
    if ((at * 8 & ((1 << p.group_shift) - 1)) == 0) store_scale(out + scale_at(p, row, at * 8 >> p.group_shift), p.s_type, scale);
  }
}

// ------------------------------------------------------------------ products
bool valid_w4_type(int32_t t) { return t == PQ_F32 || t == PQ_F16 || t == PQ_BF16; }

bool valid_w4(const pq_w4_weights* w) {
  return w != nullptr && w->N >= 1 && w->K >= 1 && w->K <= 131072 && w->N <= 0x7FFFFFF0 &&
         (w->group == 32 || w->group == 64 || w->group == 128) && valid_w4_type(w->s_type);
}

bool valid_w4_call(const pq_w4_weights* w, const pq_linear_desc* d) {
  return valid_w4(w) && d != nullptr && d->M >= 0 && d->N == w->N && d->K == w->K && valid_w4_type(d->x_type) &&
         valid_w4_type(d->y_type) && d->ldx >= d->K && d->ldy >= d->N;
}

// Whether no output lies on a token's element: apart as a whole, or columns of their own in rows of one pitch (bytes).
// (Blocks read tokens while others write outputs.)
bool rows_apart(const void* x_dev, const void* y_dev, const pq_linear_desc* d) {
  const __int128 x = static_cast<__int128>(reinterpret_cast<uintptr_t>(x_dev)), y = static_cast<__int128>(reinterpret_cast<uintptr_t>(y_dev));
  const __int128 ex = bytes_of_type(d->x_type), ey = bytes_of_type(d->y_type), px = d->ldx * ex, py = d->ldy * ey;
  if (x + (d->M - 1) * px + d->K * ex <= y || y + (d->M - 1) * py + d->N * ey <= x) return true;
  if (d->M == 1 || px != py) return false;
  const __int128 off = ((y - x) % px + px) % px;  // of y's row in x's
  return off >= d->K * ex && off + d->N * ey <= px;
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
  return static_cast<size_t>(p.strips) * static_cast<size_t>(p.blocks) * static_cast<size_t>(p.block_bytes);
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
  return pq::valid_w4_call(w, d) ? pq::w4_tc_scratch(d->M, d->N, d->K, d->ldx, d->x_type) : 0;
}

pq_status palquant_linear_w4(const void* x_dev, const void* packed_dev, const float* bias_dev, void* y_dev,
                             const pq_w4_weights* w, const pq_linear_desc* d, void* scratch_dev, size_t scratch_bytes,
                             pq_stream_t stream) {
  if (!pq::valid_w4_call(w, d)) return PQ_EINVAL;
  if (d->M == 0) return PQ_OK;
  const size_t e = pq::bytes_of_type(d->x_type);
  if (x_dev == nullptr || packed_dev == nullptr || y_dev == nullptr || !pq::is_aligned(x_dev, e) ||
      !pq::is_aligned(packed_dev, 16) || !pq::is_aligned(bias_dev, 4) || !pq::is_aligned(y_dev, pq::bytes_of_type(d->y_type)))
    return PQ_EINVAL;
  if (d->M > 32ll * 65535) return PQ_EUNSUPPORTED;  // blocks along the grid's second axis
  if (!pq::rows_apart(x_dev, y_dev, d)) return PQ_EINVAL;
  const size_t need = palquant_linear_w4_scratch_bytes(w, d);
  if (need > 0 && (scratch_dev == nullptr || scratch_bytes < need || !pq::is_aligned(scratch_dev, 16))) return PQ_EINVAL;
  const pq::W4Args a = {pq::packed_of(w), x_dev, static_cast<const uint8_t*>(packed_dev), bias_dev, y_dev, d->ldx, d->ldy, d->M,
                        d->N, d->K, d->y_type, pq::is_aligned(x_dev, 4 * e) && d->ldx % 4 == 0};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t st = pq::w4_tc_takes(a, d->x_type) ? pq::launch_w4_tc(a, d->x_type, scratch_dev, s)
                         : d->x_type == PQ_F32         ? pq::launch_w4_rows<float>(a, s)
                         : d->x_type == PQ_F16         ? pq::launch_w4_rows<__half>(a, s)
                                                       : pq::launch_w4_rows<__nv_bfloat16>(a, s);
  return st == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

}  // extern "C"
