// Norms of query and key heads and the rotation by position, in one pass.
//
// Mathematics.  For each head x of D elements: y_i = x_i w_i / sqrt(sum x^2 / D + eps), then the pairs
// (y_i, y_{i + R/2}) (or (y_2i, y_{2i+1})) of the first R elements turn by the angle pos f_i.  A frequency comes as
// a 64-bit fraction of a turn, F_i = f_i / 2 pi * 2^64 to 2 units, and pos F_i mod 2^64 is the angle's fraction of a turn, off by
// at most |pos| 2^-63 turns: whole turns fall off the top of the product.  Its nearest quarter turn is
// taken out in integers, and all 64 bits of the rest (an eighth of a turn at most) are rounded to fp32 at once: a small angle's sine
// is as exact relative to itself as a large one's.
// Everything after is fp32, rounded to the type once.
//
// Split.  Bound by HBM: each element is read and written once.  A block takes a few tokens with all their heads, so
// that a token's cosines and sines are computed once a block and not once a head; 2^k lanes hold a head,
// each two 16-byte pieces, so that both members of every pair are in one thread and the sum of squares
// needs k shuffles.  Whole heads are in registers before they are written: outputs may be the inputs.  Measured: 13003 tokens of 32 + 8
// heads of 128, bfloat16, 53 us (5.0 TB/s; a warp a head, its partners through shared memory, 404), one token 3.3.  What
// does not fit these pieces goes through pq_qk_rope_any: 13003 tokens of 32 + 8 heads of 80, 40 rotated, bfloat16, 355 us.
#include <cuda_runtime.h>

#include <cmath>

#include "palquant.h"
#include "pq_apart.h"
#include "pq_internal.h"
#include "pq_tokens.cuh"

namespace pq {
namespace {

constexpr int kThreads = 256;
constexpr int kMostD = 1024;

struct RopeArgs {
  pq_qk_rope d;
  const void* in[2];  // queries, keys
  void* out[2];
  int heads;   // of both
  int block_tokens;
  int token_groups;  // pq_qk_rope_wide: lane groups that share a token's heads
};

// cos and sin of pos * F / 2^64 turns.
__device__ __forceinline__ float2 cos_sin(int pos, uint64_t turns) {
  const uint64_t t = static_cast<uint64_t>(static_cast<int64_t>(pos)) * turns;
  const uint32_t quarter = static_cast<uint32_t>((t + (1ull << 61)) >> 62);
  // the rest, at most an eighth of a turn of either sign, rounded to fp32 once (the sine of a small angle is as exact as the angle)
  const int64_t rest = static_cast<int64_t>(t - (static_cast<uint64_t>(quarter) << 62));
  float s, c;
  sincospif(__ll2float_rn(rest) * 0x1p-63f, &s, &c);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

__device__ __forceinline__ float weight_at(const void* w, int type, int i) {
  if (w == nullptr) return 1.0f;
  if (type == PQ_F32) return static_cast<const float*>(w)[i];
  if (type == PQ_F16) return __half2float(static_cast<const __half*>(w)[i]);
  return __bfloat162float(static_cast<const __nv_bfloat16*>(w)[i]);
}

// The block's angles [tokens][R / 2] and weights [2][D], in shared memory.
__device__ __forceinline__ void block_tables(const RopeArgs& p, int64_t tok0, int tokens, float2* angles, float* weights) {
  const int half = p.d.R / 2;
  for (int i = threadIdx.x; i < tokens * half; i += blockDim.x) {
    const int t = i / half;
    angles[i] = cos_sin(p.d.pos_dev[tok0 + t], p.d.turns_dev[i - t * half]);
  }
  if (p.d.norm)
    for (int i = threadIdx.x; i < 2 * p.d.D; i += blockDim.x)
      weights[i] = i < p.d.D ? weight_at(p.d.q_weight_dev, p.d.w_type, i) : weight_at(p.d.k_weight_dev, p.d.w_type, i - p.d.D);
}

template <typename T>
__device__ __forceinline__ T* head_at(const RopeArgs& p, const void* base, int64_t token, int head, bool key, bool out) {
  const int64_t ts = out ? (key ? p.d.k_out_token_stride : p.d.q_out_token_stride) : (key ? p.d.k_token_stride : p.d.q_token_stride);
  const int64_t hs = out ? (key ? p.d.k_out_head_stride : p.d.q_out_head_stride) : (key ? p.d.k_head_stride : p.d.q_head_stride);
  return static_cast<T*>(const_cast<void*>(base)) + token * ts + head * hs;
}

// Any D up to kMostD, any alignment: a warp a head, pairs and single elements spread over its lanes.
template <typename T>
__global__ void __launch_bounds__(kThreads) pq_qk_rope_any(const __grid_constant__ RopeArgs p) {
  extern __shared__ float2 tables[];
  const int D = p.d.D, half = p.d.R / 2, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t tok0 = static_cast<int64_t>(blockIdx.x) * p.block_tokens;
  const int tokens = static_cast<int>(min(static_cast<int64_t>(p.block_tokens), p.d.tokens - tok0));
  float* weights = reinterpret_cast<float*>(tables + p.block_tokens * half);
  block_tables(p, tok0, tokens, tables, weights);
  __syncthreads();
  for (int item = warp; item < tokens * p.heads; item += kThreads / 32) {
    const int t = item / p.heads, h = item - t * p.heads;
    const bool key = h >= p.d.Hq;
    const T* src = head_at<T>(p, p.in[key], tok0 + t, key ? h - p.d.Hq : h, key, false);
    T* dst = head_at<T>(p, p.out[key], tok0 + t, key ? h - p.d.Hq : h, key, true);
    float x[kMostD / 32];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kMostD / 32; ++i) {
      const int d = lane + 32 * i;
      x[i] = d < D ? to_f32(src[d]) : 0.0f;
      sum = fmaf(x[i], x[i], sum);
    }
    float f = 1.0f;
    if (p.d.norm) {
#pragma unroll
      for (int s = 16; s > 0; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
      f = __frsqrt_rn(sum / static_cast<float>(D) + p.d.eps);
    }
    __syncwarp();  // the head is in registers: the output may lie where it was
    const float* w = weights + (key ? D : 0);
    const float2* angle = tables + t * half;
    // each element's partner sits in another lane's registers: it is read again from the normed values in shared memory
    float* row = weights + (p.d.norm ? 2 * D : 0) + warp * D;
#pragma unroll
    for (int i = 0; i < kMostD / 32; ++i) {
      const int d = lane + 32 * i;
      if (d < D) row[d] = p.d.norm ? x[i] * f * w[d] : x[i];
    }
    __syncwarp();
    for (int d = lane; d < D; d += 32) {
      float y = row[d];
      if (d < p.d.R) {
        const int pair = p.d.interleaved ? d >> 1 : d < half ? d : d - half;
        const bool second = p.d.interleaved ? d & 1 : d >= half;
        const float other = row[p.d.interleaved ? d ^ 1 : second ? d - half : d + half];
        const float2 cs = angle[pair];
        y = second ? fmaf(y, cs.x, other * cs.y) : fmaf(y, cs.x, -other * cs.y);
      }
      dst[d] = from_f32<T>(y);
    }
    __syncwarp();
  }
}

// Heads on 16-byte boundaries whose pairs fill 16-byte pieces: 2^LG lanes hold a head, lane u the pieces first(u) and
// second(u).  A group of lanes keeps a token's cosines and sines in registers while it goes through heads of that token, the next
// head on its way before the last one is written.
template <typename T, int LG>
__global__ void __launch_bounds__(kThreads) pq_qk_rope_wide(const __grid_constant__ RopeArgs p) {
  constexpr int V = 16 / sizeof(T);  // elements of a piece
  constexpr int kLanes = 1 << LG;
  extern __shared__ float2 tables[];
  const int D = p.d.D, R = p.d.R, half = R / 2;
  const int u = threadIdx.x & (kLanes - 1), group = threadIdx.x >> LG;
  const int64_t tok0 = static_cast<int64_t>(blockIdx.x) * p.block_tokens;
  const int tokens = static_cast<int>(min(static_cast<int64_t>(p.block_tokens), p.d.tokens - tok0));
  const int t = group / p.token_groups;
  const bool there = u < D / (2 * V) && t < tokens;
  const int rotated = R / (2 * V);  // lanes whose pieces are partners
  const int first = p.d.interleaved ? 2 * u * V : u < rotated ? u * V : R + 2 * (u - rotated) * V;
  const int second = p.d.interleaved || u >= rotated ? first + V : half + u * V;
  auto at = [&](int h, bool out) {
    const bool key = h >= p.d.Hq;
    return head_at<T>(p, (out ? p.out : p.in)[key], tok0 + t, key ? h - p.d.Hq : h, key, out);
  };
  int h = group % p.token_groups;
  uint4 next[2];
  if (there && h < p.heads) {
    const T* src = at(h, false);
    next[0] = *reinterpret_cast<const uint4*>(src + first);
    next[1] = *reinterpret_cast<const uint4*>(src + second);
  }
  float* weights = reinterpret_cast<float*>(tables + p.block_tokens * half);
  block_tables(p, tok0, tokens, tables, weights);
  __syncthreads();
  // angles of this lane's pairs: V of two pieces, or V / 2 of each
  float2 cs[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int pair = u * V + i;
    cs[i] = there && pair < half && (p.d.interleaved || u < rotated) ? tables[t * half + pair] : make_float2(1.0f, 0.0f);
  }
  float w[2][V];
  int weights_of = -1;
  // (as often for every group of the warp: they sum together)
  for (int turns = (p.heads + p.token_groups - 1) / p.token_groups; turns > 0; --turns, h += p.token_groups) {
    const bool head = there && h < p.heads;
    const uint4 now[2] = {next[0], next[1]};
    if (there && h + p.token_groups < p.heads) {
      const T* src = at(h + p.token_groups, false);
      next[0] = *reinterpret_cast<const uint4*>(src + first);
      next[1] = *reinterpret_cast<const uint4*>(src + second);
    }
    float x[2][V];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      T raw[V];
      memcpy(raw, &now[j], 16);
#pragma unroll
      for (int i = 0; i < V; ++i) x[j][i] = head ? to_f32(raw[i]) : 0.0f;
    }
    if (p.d.norm) {
      const int key = h >= p.d.Hq;
      if (key != weights_of) {
        weights_of = key;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          w[0][i] = there ? weights[key * D + first + i] : 0.0f;
          w[1][i] = there ? weights[key * D + second + i] : 0.0f;
        }
      }
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) sum = fmaf(x[0][i], x[0][i], fmaf(x[1][i], x[1][i], sum));
#pragma unroll
      for (int s = kLanes / 2; s > 0; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s, kLanes);
      const float f = __frsqrt_rn(sum / static_cast<float>(D) + p.d.eps);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) x[j][i] = x[j][i] * f * w[j][i];
    }
    T y[2][V];
    // (elements behind the rotated part are taken as they are: times (1, 0) an infinity would make its neighbour NaN)
    if (p.d.interleaved) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < V; i += 2) {
          const float2 c = cs[(j * V + i) / 2];
          const bool turned = u * V + (j * V + i) / 2 < half;
          y[j][i] = from_f32<T>(turned ? fmaf(x[j][i], c.x, -x[j][i + 1] * c.y) : x[j][i]);
          y[j][i + 1] = from_f32<T>(turned ? fmaf(x[j][i + 1], c.x, x[j][i] * c.y) : x[j][i + 1]);
        }
    } else {
      const bool turned = u < rotated;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        y[0][i] = from_f32<T>(turned ? fmaf(x[0][i], cs[i].x, -x[1][i] * cs[i].y) : x[0][i]);
        y[1][i] = from_f32<T>(turned ? fmaf(x[1][i], cs[i].x, x[0][i] * cs[i].y) : x[1][i]);
      }
    }
    if (head) {
      T* dst = at(h, true);
      uint4 out[2];
      memcpy(out, y, 32);
      *reinterpret_cast<uint4*>(dst + first) = out[0];
      *reinterpret_cast<uint4*>(dst + second) = out[1];
    }
  }
}

int64_t any_smem(const RopeArgs& p) {
  return static_cast<int64_t>(p.block_tokens) * (p.d.R / 2) * 8 + (p.d.norm ? 2 : 0) * p.d.D * 4 + static_cast<int64_t>(kThreads / 32) * p.d.D * 4;
}

// Rows of 16-byte pieces whose pairs share pieces or lie in two that one lane takes.
template <typename T>
bool takes_wide(const RopeArgs& p) {
  constexpr int V = 16 / sizeof(T);
  const pq_qk_rope& d = p.d;
  if (d.D % (2 * V) != 0 || d.D > 64 * V || (!d.interleaved && d.R % (2 * V) != 0)) return false;
  for (int key = 0; key < 2; ++key)
    if ((key ? d.Hkv : d.Hq) > 0 && (!is_aligned(p.in[key], 16) || !is_aligned(p.out[key], 16))) return false;
  for (int64_t s : {d.q_token_stride, d.q_head_stride, d.q_out_token_stride, d.q_out_head_stride})
    if (d.Hq > 0 && s % V != 0) return false;
  for (int64_t s : {d.k_token_stride, d.k_head_stride, d.k_out_token_stride, d.k_out_head_stride})
    if (d.Hkv > 0 && s % V != 0) return false;
  return true;
}

template <typename T>
cudaError_t launch_wide(RopeArgs& p, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  int lg = 0;
  while ((2 * V << lg) < p.d.D) ++lg;
  const int groups = kThreads >> lg;
  // about ten heads a group (13003 tokens of 32 + 8 heads of 128: 52.4 us; five 54.6, twenty 54.4); a group for each head where the tokens
  // would not fill the chip
  int share = 1;
  while (share < groups && share * 10 < p.heads) share *= 2;
  while (share < groups && share < p.heads && p.d.tokens * share < 304ll * groups) share *= 2;
  p.token_groups = share;
  p.block_tokens = groups / share;
  const unsigned blocks = static_cast<unsigned>((p.d.tokens + p.block_tokens - 1) / p.block_tokens);
  const size_t smem = static_cast<size_t>(p.block_tokens) * (p.d.R / 2) * 8 + (p.d.norm ? 2 * p.d.D * 4 : 0);
  switch (lg) {
    case 0: pq_qk_rope_wide<T, 0><<<blocks, kThreads, smem, s>>>(p); break;
    case 1: pq_qk_rope_wide<T, 1><<<blocks, kThreads, smem, s>>>(p); break;
    case 2: pq_qk_rope_wide<T, 2><<<blocks, kThreads, smem, s>>>(p); break;
    case 3: pq_qk_rope_wide<T, 3><<<blocks, kThreads, smem, s>>>(p); break;
    case 4: pq_qk_rope_wide<T, 4><<<blocks, kThreads, smem, s>>>(p); break;
    default: pq_qk_rope_wide<T, 5><<<blocks, kThreads, smem, s>>>(p); break;
  }
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_rope(RopeArgs& p, cudaStream_t s) {
  if (takes_wide<T>(p)) return launch_wide<T>(p, s);
  p.block_tokens = 1;
  const int64_t blocks = (p.d.tokens + p.block_tokens - 1) / p.block_tokens;
  pq_qk_rope_any<T><<<static_cast<unsigned>(blocks), kThreads, any_smem(p), s>>>(p);
  return cudaGetLastError();
}

// The fraction of a number of turns, in units of 2^-64.
uint64_t fraction(double turns) {
  if (std::fabs(turns) < 0.25) return static_cast<uint64_t>(std::llrint(turns * 0x1p64));  // (modulo 2^64 below 0)
  const double f = turns - std::floor(turns);
  return f < 1.0 ? static_cast<uint64_t>(f * 0x1p64) : 0;
}

bool valid_rope(const pq_qk_rope* d) {
  if (d == nullptr) return false;
  auto type = [](int32_t t) { return t == PQ_F32 || t == PQ_F16 || t == PQ_BF16; };
  if (!type(d->type) || d->tokens < 0 || d->Hq < 0 || d->Hkv < 0 || d->Hq + static_cast<int64_t>(d->Hkv) < 1 || d->D < 1) return false;
  if (d->R < 0 || d->R > d->D || d->R % 2 != 0) return false;
  if ((d->interleaved != 0 && d->interleaved != 1) || (d->norm != 0 && d->norm != 1)) return false;
  if (d->norm && (!type(d->w_type) || !(d->eps >= 0.0f) || d->eps == INFINITY)) return false;
  for (int64_t s : {d->q_token_stride, d->q_head_stride, d->k_token_stride, d->k_head_stride, d->q_out_token_stride,
                    d->q_out_head_stride, d->k_out_token_stride, d->k_out_head_stride})
    if (s < 0) return false;
  return true;
}

// Whether no output lies on an element of another tensor: each is its input itself, or shares nothing with it, and nothing with the others.
// (A head is written while others are still to be read.)
bool outputs_apart(const RopeArgs& p) {
  const pq_qk_rope& d = p.d;
  const __int128 e = static_cast<__int128>(bytes_of_type(d.type));
  auto heads = [&](const void* at, int64_t ts, int64_t hs, int n) { return HeadsAt{reinterpret_cast<uintptr_t>(at), ts * e, hs * e, n}; };
  const HeadsAt in[2] = {heads(p.in[0], d.q_token_stride, d.q_head_stride, d.Hq), heads(p.in[1], d.k_token_stride, d.k_head_stride, d.Hkv)};
  const HeadsAt out[2] = {heads(p.out[0], d.q_out_token_stride, d.q_out_head_stride, d.Hq),
                          heads(p.out[1], d.k_out_token_stride, d.k_out_head_stride, d.Hkv)};
  const int64_t bytes = d.D * static_cast<int64_t>(e);
  for (int o = 0; o < 2; ++o)
    for (int i = 0; i < 2; ++i)
      if (!(o == i && same_heads(out[o], in[i], d.tokens)) && heads_share(out[o], in[i], d.tokens, bytes)) return false;
  return !heads_share(out[0], out[1], d.tokens, bytes);
}

}  // namespace
}  // namespace pq

extern "C" {

pq_status palquant_rope_turns_host(const double* frequencies_host, int32_t n, uint64_t* turns_host) {
  if (n < 0 || (n > 0 && (frequencies_host == nullptr || turns_host == nullptr))) return PQ_EINVAL;
  for (int32_t i = 0; i < n; ++i) {
    if (!std::isfinite(frequencies_host[i])) return PQ_EINVAL;
  }
  for (int32_t i = 0; i < n; ++i) {
    // f / 2 pi with its rounding's rest (the reciprocal in two doubles), the fraction of each as 2^-64 turns
    const double f = frequencies_host[i], inv = 0x1.45f306dc9c883p-3, inv_rest = -0x1.6b01ec5417056p-57;
    const double turns = f * inv, rest = std::fma(f, inv, -turns) + f * inv_rest;
    turns_host[i] = pq::fraction(turns) + pq::fraction(rest);  // modulo 2^64: whole turns
  }
  return PQ_OK;
}

pq_status palquant_qk_norm_rope(const void* q_dev, const void* k_dev, void* q_out_dev, void* k_out_dev, const pq_qk_rope* d,
                                pq_stream_t stream) {
  using namespace pq;
  if (!valid_rope(d)) return PQ_EINVAL;
  if (d->tokens == 0) return PQ_OK;
  const size_t e = bytes_of_type(d->type);
  if (d->Hq > 0 && (q_dev == nullptr || q_out_dev == nullptr || !is_aligned(q_dev, e) || !is_aligned(q_out_dev, e))) return PQ_EINVAL;
  if (d->Hkv > 0 && (k_dev == nullptr || k_out_dev == nullptr || !is_aligned(k_dev, e) || !is_aligned(k_out_dev, e))) return PQ_EINVAL;
  if (d->R > 0 && (d->pos_dev == nullptr || d->turns_dev == nullptr || !is_aligned(d->pos_dev, 4) || !is_aligned(d->turns_dev, 8)))
    return PQ_EINVAL;
  if (d->norm && (!is_aligned(d->q_weight_dev, bytes_of_type(d->w_type)) || !is_aligned(d->k_weight_dev, bytes_of_type(d->w_type))))
    return PQ_EINVAL;
  if (d->D > kMostD || d->tokens > 0x7FFFFFFF || d->Hq + static_cast<int64_t>(d->Hkv) > 65535) return PQ_EUNSUPPORTED;
  RopeArgs p = {*d, {q_dev, k_dev}, {q_out_dev, k_out_dev}, d->Hq + d->Hkv, 1, 1};
  if (!outputs_apart(p)) return PQ_EINVAL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t st = d->type == PQ_F32   ? launch_rope<float>(p, s)
                         : d->type == PQ_F16 ? launch_rope<__half>(p, s)
                                             : launch_rope<__nv_bfloat16>(p, s);
  return st == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

}  // extern "C"
