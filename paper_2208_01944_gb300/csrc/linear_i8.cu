// Dense layers on signed 8-bit codes, y = (q W^T) s_x s_w + bias, and the token
// quantiser before them.
//
// pq_quantize_tokens: one block per token; the token stays in registers between
// the search for its largest magnitude and the rounding (one read of x, one write
// of the codes; HBM-bound).
//
// pq_linear_rows: any size, any alignment; pq_linear_stream: up to 16 tokens on 16-byte
// boundaries, the same work out of rings of asynchronous copies.  The kernels of few tokens, where the
// weights' bytes are what counts.  mma.sync on 8-bit integers runs at 158 TOPS on
// this chip, far below the half-precision rate, and 8-bit codes are exact half
// values, so the codes are turned into halves in registers (1.25 instructions a
// code) and multiplied with fp32 sums.  Those are exact as long as they stay below 2^24:
// 127 * 128 * 1024 = 16646144 < 2^24, so every warp adds its fp32 sums to int32
// ones after at most 1024 of K.  The weights are the 16-row operand of the MMA and
// the tokens its 8 columns, so few tokens waste little.  The warps of a block share
// 16 output channels and take turns along K, each lane reading 16 contiguous
// bytes; within a 64-wide step the order of K is the lanes' own, the same for both
// operands.  Measured, whole calls in a graph, inputs in turn beyond L2: one token times 4096 x 4096 7.5 us, 8 x
// 8192 x 8192 17.2 us (3.9 TB/s of weights), one token times 12000 rows of 1001 codes 9.4 us.
#include <cuda_runtime.h>

#include <algorithm>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_linear.h"
#include "pq_tokens.cuh"
#include "pq_words.h"

namespace pq {
namespace {

constexpr int kTokThreads = 256;

// NV: vectors of 8 elements that a thread keeps; 0: the token is read twice.
template <typename T, bool HALF, int NV>
__global__ void __launch_bounds__(kTokThreads) pq_quantize_tokens(const T* __restrict__ x, int64_t ldx, int K,
                                                                  void* __restrict__ q, int64_t ldq,
                                                                  float* __restrict__ s, bool wide_x, bool wide_q) {
  __shared__ uint32_t red[8];
  const int64_t m = blockIdx.x;
  const T* row = x + m * ldx;
  const int nvec = (K + 7) / 8;
  let_next_kernel_start();
  Vec8<T> keep[NV > 0 ? NV : 1];
  uint32_t top = 0;
  if (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = threadIdx.x + i * blockDim.x;
      if (v < nvec) keep[i] = load8(row + 8 * v, K - 8 * v, wide_x && 8 * v + 8 <= K);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (threadIdx.x + i * blockDim.x < nvec) top = max(top, amax8(keep[i]));
  } else {
    for (int v = threadIdx.x; v < nvec; v += blockDim.x)
      top = max(top, amax8(load8(row + 8 * v, K - 8 * v, wide_x && 8 * v + 8 <= K)));
  }
  top = block_max(top, red);
  const float scale = scale_of_amax(top), inv = inverse_of_scale(scale);
  if (threadIdx.x == 0) s[m] = scale;
  auto put = [&](int v, const Vec8<T>& r) {
    const int left = K - 8 * v;
    const bool wide = wide_q && left >= 8;
    if (HALF) {
      store8(static_cast<__half*>(q) + m * ldq + 8 * v, half_codes8(r, inv), left, wide);
    } else {
      const uint2 c = codes8(r, inv);
      int8_t* dst = static_cast<int8_t*>(q) + m * ldq + 8 * v;
      if (wide) {
        *reinterpret_cast<uint2*>(dst) = c;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < left) dst[i] = static_cast<int8_t>((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
      }
    }
  };
  if (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = threadIdx.x + i * blockDim.x;
      if (v < nvec) put(v, keep[i]);
    }
  } else {
    for (int v = threadIdx.x; v < nvec; v += blockDim.x)
      put(v, load8(row + 8 * v, K - 8 * v, wide_x && 8 * v + 8 <= K));
  }
}

template <typename T, bool HALF>
cudaError_t launch_tokens(const void* x, int64_t ldx, int64_t M, int K, void* q, int64_t ldq, float* s,
                          cudaStream_t stream) {
  const bool wide_x = is_aligned(x, 16) && ldx * sizeof(T) % 16 == 0;
  const size_t qe = HALF ? 2 : 1;
  const bool wide_q = is_aligned(q, 8 * qe) && ldq % 8 == 0;
  const int nvec = (K + 7) / 8;
  const int threads = std::min(kTokThreads, (nvec + 31) / 32 * 32);
  const int nv = (nvec + threads - 1) / threads;
  const T* xt = static_cast<const T*>(x);
  const unsigned grid = static_cast<unsigned>(M);
  if (nv <= 1)
    pq_quantize_tokens<T, HALF, 1><<<grid, threads, 0, stream>>>(xt, ldx, K, q, ldq, s, wide_x, wide_q);
  else if (nv <= 2)
    pq_quantize_tokens<T, HALF, 2><<<grid, threads, 0, stream>>>(xt, ldx, K, q, ldq, s, wide_x, wide_q);
  else if (nv <= 4)
    pq_quantize_tokens<T, HALF, 4><<<grid, threads, 0, stream>>>(xt, ldx, K, q, ldq, s, wide_x, wide_q);
  else if (nv <= 8)
    pq_quantize_tokens<T, HALF, 8><<<grid, threads, 0, stream>>>(xt, ldx, K, q, ldq, s, wide_x, wide_q);
  else
    pq_quantize_tokens<T, HALF, 0><<<grid, threads, 0, stream>>>(xt, ldx, K, q, ldq, s, wide_x, wide_q);
  return cudaGetLastError();
}

// ------------------------------------------------------------------ products
// 16 codes of a row from column k on as bytes, zeros past K.  Rows that no 16-byte load
// may read come in aligned words, shifted together, as long as those lie inside the row.
template <bool WIDE>
__device__ __forceinline__ uint4 codes16(const int8_t* row, int k, int K) {
  if (WIDE && k + 16 <= K) return *reinterpret_cast<const uint4*>(row + k);
  uint32_t w[4] = {0, 0, 0, 0};
  const uintptr_t at = reinterpret_cast<uintptr_t>(row + k);
  if (!WIDE && words_lie_in_row(k, K, static_cast<int>(at & 3))) {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(at & ~static_cast<uintptr_t>(3));
    const unsigned shift = 8 * static_cast<unsigned>(at & 3);
    const uint32_t a = p[0], b = p[1], c = p[2], d = p[3], e = p[4];
    return make_uint4(__funnelshift_r(a, b, shift), __funnelshift_r(b, c, shift), __funnelshift_r(c, d, shift),
                      __funnelshift_r(d, e, shift));
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (k + i < K) w[i >> 2] |= static_cast<uint32_t>(static_cast<uint8_t>(row[k + i])) << (8 * (i & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The same 16 columns of a token: bytes, or halves.
template <bool HALF>
__device__ __forceinline__ void load_tokens(const void* q, int64_t row, int k, int K, bool wide,
                                            uint32_t (&r)[HALF ? 8 : 4]) {
  if constexpr (HALF) {
    const __half* p = static_cast<const __half*>(q) + row + k;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const Vec8<__half> v = load8(p + 8 * j, K - k - 8 * j, wide && k + 8 * j + 8 <= K);
      memcpy(r + 4 * j, &v, sizeof(v));
    }
  } else {
    const int8_t* p = static_cast<const int8_t*>(q) + row;
    const uint4 u = wide ? codes16<true>(p, k, K) : codes16<false>(p, k, K);
    r[0] = u.x, r[1] = u.y, r[2] = u.z, r[3] = u.w;
  }
}

// Weight rows that lie off 16-byte boundaries, copied to rows of `pitch` bytes (a multiple
// of 16; zeros past K) for the tensor cores' loads.  Bound by the bytes.
__global__ void __launch_bounds__(256) pq_align_weights(const int8_t* __restrict__ w, int64_t ldw, int N, int K,
                                                        int8_t* __restrict__ out, int64_t pitch) {
  const int pieces = static_cast<int>(pitch / 16);
  const int64_t total = static_cast<int64_t>(N) * pieces, step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += step) {
    const int64_t n = i / pieces;
    const int k = static_cast<int>(i - n * pieces) * 16;
    *reinterpret_cast<uint4*>(out + n * pitch + k) = codes16<false>(w + n * ldw, k, K);
  }
}

constexpr int kRowWarps = 8;
constexpr int kExactSteps = 16;  // 64-wide steps whose fp32 sums are exact
constexpr int kAhead = 2;        // (four took the registers of a fourth block on an SM)
static_assert(kExactSteps % kAhead == 0, "sums are moved between rounds of kAhead steps");

// The warps' sums of a block's 16 channels x 8 NT tokens, added and written.
template <int NT>
__device__ __forceinline__ void put_parts(const LinearArgs& a, int32_t (&part)[kRowWarps][NT][8][17],
                                          const int32_t (&sum)[NT][4], int n0, int64_t m0) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[warp][j][2 * t + (e & 1)][g + 8 * (e >> 1)] = sum[j][e];
  __syncthreads();
  for (int e = threadIdx.x; e < NT * 128; e += 32 * kRowWarps) {
    const int r = e & 15, c = (e >> 4) & 7, j = e >> 7;
    const int n = n0 + r;
    const int64_t m = m0 + 8 * j + c;
    if (n >= a.N || m >= a.M) continue;
    const float s_x = a.s_x != nullptr ? a.s_x[m] : 0.0f, s_w = a.s_w != nullptr ? a.s_w[n] : 0.0f;
    const float bias = a.bias != nullptr ? a.bias[n] : 0.0f;
    int32_t acc = 0;
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) acc += part[w][j][c][r];
    put_result(a, m, n, acc, s_x, s_w, bias);
  }
}

// A block: 16 output channels x 8 NT tokens.
template <int NT, bool HALF, bool WIDE>
__global__ void __launch_bounds__(32 * kRowWarps) pq_linear_rows(const __grid_constant__ LinearArgs a) {
  __shared__ int32_t part[kRowWarps][NT][8][17];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * 16;
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * (8 * NT);
  const int steps = (a.K + 63) / 64;
  // rows past the end read the last row again; their sums are not stored
  const int8_t* w0 = a.w + static_cast<int64_t>(min(n0 + g, a.N - 1)) * a.ldw;
  const int8_t* w1 = a.w + static_cast<int64_t>(min(n0 + g + 8, a.N - 1)) * a.ldw;
  int64_t tok[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) tok[j] = min(m0 + 8 * j + g, a.M - 1) * a.ldq;

  // a round is kAhead steps, all loaded before the first is multiplied; the first round's
  // weights come before the kernel that writes the tokens' codes is over
  uint4 u[kAhead][2];
  auto load_w = [&](int s0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int s = s0 + i * kRowWarps, k = s * 64 + t * 16;
      if (s < steps) {
        u[i][0] = codes16<WIDE>(w0, k, a.K);
        u[i][1] = codes16<WIDE>(w1, k, a.K);
      }
    }
  };
  load_w(warp);
  wait_previous_kernel();
  int32_t sum[NT][4] = {};
  float d[NT][4] = {};
  int done = 0;  // steps in the fp32 sums
  for (int s0 = warp; s0 < steps; s0 += kAhead * kRowWarps) {
    if (s0 != warp) load_w(s0);
    uint32_t b[kAhead][NT][HALF ? 8 : 4];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int s = s0 + i * kRowWarps, k = s * 64 + t * 16;
      if (s < steps) {
#pragma unroll
        for (int j = 0; j < NT; ++j) load_tokens<HALF>(a.q, tok[j], k, a.K, a.wide_q, b[i][j]);
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (s0 + i * kRowWarps >= steps) break;
      const uint32_t x0[4] = {u[i][0].x, u[i][0].y, u[i][0].z, u[i][0].w};
      const uint32_t x1[4] = {u[i][1].x, u[i][1].y, u[i][1].z, u[i][1].w};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t r0, r1, r2, r3;
        half_of_codes(x0[c], r0, r2);
        half_of_codes(x1[c], r1, r3);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          uint32_t b0, b1;
          if constexpr (HALF)
            b0 = b[i][j][2 * c], b1 = b[i][j][2 * c + 1];
          else
            half_of_codes(b[i][j][c], b0, b1);
          mma_16x8x16(d[j], r0, r1, r2, r3, b0, b1);
        }
      }
    }
    done += kAhead;
    if (done == kExactSteps || s0 + kAhead * kRowWarps >= steps) {
      done = 0;
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[j][e] += __float2int_rn(d[j][e]), d[j][e] = 0.0f;
    }
  }
  put_parts<NT>(a, part, sum, n0, m0);
}

// The same product for weights and 8-bit tokens whose rows lie on 16-byte boundaries: every
// lane copies the pieces it will multiply into shared memory of its own, RING - 1 steps
// ahead (no other lane reads them, so nothing but the lane's own copies is waited for).
// Bound by the weights' bytes; registers hold one step, so blocks of 8 warps keep 100 KB in
// flight on an SM.  The rings are no deeper than a warp has steps, for more blocks on an SM
// where K is short.  When they came, calls with their weights in L2 (now 6.1 and 15.4 us): one token times 4096 x 4096
// 9.8 us with loads into registers, 6.5 with these rings, 7.0 with rings of 8 steps; 8 x 8192 x 8192 20.7, 17.3 and 18.5.
template <int NT, int RING>
__host__ __device__ constexpr int ring_bytes() { return kRowWarps * RING * (2 + NT) * 512; }

template <int NT, int RING>
__global__ void __launch_bounds__(32 * kRowWarps) pq_linear_stream(const __grid_constant__ LinearArgs a) {
  constexpr int kRing = RING, kStep = (2 + NT) * 512;
  extern __shared__ __align__(16) uint8_t ring_raw[];
  __shared__ int32_t part[kRowWarps][NT][8][17];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * 16;
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * (8 * NT);
  const int steps = (a.K + 63) / 64, mine = steps > warp ? (steps - warp - 1) / kRowWarps + 1 : 0;
  // rows past the end read the last row again; their sums are not stored
  const int8_t* w0 = a.w + static_cast<int64_t>(min(n0 + g, a.N - 1)) * a.ldw;
  const int8_t* w1 = a.w + static_cast<int64_t>(min(n0 + g + 8, a.N - 1)) * a.ldw;
  const int8_t* tok[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) tok[j] = static_cast<const int8_t*>(a.q) + min(m0 + 8 * j + g, a.M - 1) * a.ldq;
  // tokens past the end are zeros and read nothing: every block reads the same few lines of
  // tokens, and eight lanes asking for one line of a single token made 1 x 1008 x 12000 take
  // 14 us, not 4
  bool there[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) there[j] = m0 + 8 * j + g < a.M;
  const uint32_t ring = smem_u32(ring_raw) + warp * kRing * kStep + lane * 16;
  // step i of this warp: columns from k on, `left` bytes of them (the copy zeroes the rest)
  auto fetch_w = [&](int i) {
    const int k = (warp + i * kRowWarps) * 64 + t * 16, left = max(0, min(16, a.K - k)), at = left > 0 ? k : 0;
    const uint32_t to = ring + (i % kRing) * kStep;
    cp_async_16(to, w0 + at, left);
    cp_async_16(to + 512, w1 + at, left);
  };
  auto fetch_tokens = [&](int i) {
    const int k = (warp + i * kRowWarps) * 64 + t * 16, left = max(0, min(16, a.K - k)), at = left > 0 ? k : 0;
    const uint32_t to = ring + (i % kRing) * kStep + 1024;
#pragma unroll
    for (int j = 0; j < NT; ++j) cp_async_16(to + 512 * j, tok[j] + at, there[j] ? left : 0);
  };
  // the first weights come before the kernel that writes the tokens' codes is over
#pragma unroll
  for (int i = 0; i < kRing - 1; ++i)
    if (i < mine) fetch_w(i);
  wait_previous_kernel();
#pragma unroll
  for (int i = 0; i < kRing - 1; ++i) {
    if (i < mine) fetch_tokens(i);
    cp_async_commit();
  }
  int32_t sum[NT][4] = {};
  float d[NT][4] = {};
  for (int i = 0; i < mine; ++i) {
    cp_async_wait<kRing - 2>();
    const uint32_t at = ring + (i % kRing) * kStep;
    uint4 u0, u1, b[NT];
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(u0.x), "=r"(u0.y), "=r"(u0.z), "=r"(u0.w) : "r"(at) : "memory");
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(u1.x), "=r"(u1.y), "=r"(u1.z), "=r"(u1.w) : "r"(at + 512) : "memory");
#pragma unroll
    for (int j = 0; j < NT; ++j)
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                   : "=r"(b[j].x), "=r"(b[j].y), "=r"(b[j].z), "=r"(b[j].w)
                   : "r"(at + 1024 + 512 * j)
                   : "memory");
    // into the place of the step before, which this lane has read
    if (i + kRing - 1 < mine) {
      fetch_w(i + kRing - 1);
      fetch_tokens(i + kRing - 1);
    }
    cp_async_commit();
    const uint32_t x0[4] = {u0.x, u0.y, u0.z, u0.w}, x1[4] = {u1.x, u1.y, u1.z, u1.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint32_t r0, r1, r2, r3;
      half_of_codes(x0[c], r0, r2);
      half_of_codes(x1[c], r1, r3);
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const uint32_t y[4] = {b[j].x, b[j].y, b[j].z, b[j].w};
        uint32_t b0, b1;
        half_of_codes(y[c], b0, b1);
        mma_16x8x16(d[j], r0, r1, r2, r3, b0, b1);
      }
    }
    if ((i + 1) % kExactSteps == 0 || i + 1 == mine) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[j][e] += __float2int_rn(d[j][e]), d[j][e] = 0.0f;
    }
  }
  put_parts<NT>(a, part, sum, n0, m0);
}

template <int NT, bool HALF, bool WIDE>
cudaError_t launch_rows_as(const LinearArgs& a, bool after_tokens, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.N + 15) / 16), static_cast<unsigned>((a.M + 8 * NT - 1) / (8 * NT)));
  cfg.blockDim = dim3(32 * kRowWarps);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = after_tokens ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, pq_linear_rows<NT, HALF, WIDE>, a);
}

template <int NT, int RING>
cudaError_t launch_stream_as(const LinearArgs& a, bool after_tokens, cudaStream_t stream) {
  static int attr_set[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(pq_linear_stream<NT, RING>, cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes<NT, RING>());
    if (e != cudaSuccess) return e;
    if (dev < 64) attr_set[dev] = 1;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.N + 15) / 16), static_cast<unsigned>((a.M + 8 * NT - 1) / (8 * NT)));
  cfg.blockDim = dim3(32 * kRowWarps);
  cfg.dynamicSmemBytes = ring_bytes<NT, RING>();
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = after_tokens ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, pq_linear_stream<NT, RING>, a);
}

template <int NT>
cudaError_t launch_stream(const LinearArgs& a, bool after_tokens, cudaStream_t stream) {
  if (a.K <= 64 * kRowWarps) return launch_stream_as<NT, 2>(a, after_tokens, stream);
  if (a.K <= 128 * kRowWarps) return launch_stream_as<NT, 3>(a, after_tokens, stream);
  return launch_stream_as<NT, NT == 1 ? 5 : 4>(a, after_tokens, stream);
}

template <bool HALF, bool WIDE>
cudaError_t launch_rows(const LinearArgs& a, bool after_tokens, cudaStream_t stream) {
  if (a.M <= 8) return launch_rows_as<1, HALF, WIDE>(a, after_tokens, stream);
  return launch_rows_as<2, HALF, WIDE>(a, after_tokens, stream);
}

bool valid_type(int32_t t) { return t == PQ_F32 || t == PQ_F16 || t == PQ_BF16; }

bool valid_linear(const pq_linear_desc* d) {
  return d != nullptr && d->M >= 0 && d->N >= 1 && d->K >= 1 && d->K <= 131072 && valid_type(d->x_type) &&
         valid_type(d->y_type) && d->ldx >= d->K && d->ldw >= d->K && d->ldy >= d->N;
}

constexpr int64_t kMostTokens = 0x7FFFFFFF;  // a block each in the quantiser

bool aligned_rows(const pq_linear_desc* d) { return d->ldw % 16 == 0; }
// Weight rows off 16-byte boundaries: the kernels for few tokens read them in place, again for
// every 16 tokens; the tensor cores' loads want a copy.  With the copy against without (us):
// 16 x 4001 x 4000 17.0 / 11.8, 24 x 4001 x 4000 17.5 / 23.0, 512 x 4001 x 4000 30 / 200,
// 128 x 777 x 1001 14.9 / 8.5, 512 x 777 x 1001 15.3 / 19.9.
bool copies_weights(const pq_linear_desc* d) {
  return !aligned_rows(d) && d->M > 16 && static_cast<double>(d->M) * d->N * d->K >= 268435456.0;
}
int32_t q8_format(const pq_linear_desc* d) {
  return copies_weights(d) ? PQ_CODES_F16 : palquant_linear_code_format(d);
}

// The scratch: codes (rows padded to 16 elements), scales, and where it is made the copy
// of the weights (rows padded to 16 bytes); each part starts on 16 bytes.
int64_t padded_k(const pq_linear_desc* d) { return (static_cast<int64_t>(d->K) + 15) / 16 * 16; }
size_t scales_at(const pq_linear_desc* d) {
  return static_cast<size_t>(d->M) * static_cast<size_t>(padded_k(d)) * (q8_format(d) == PQ_CODES_F16 ? 2 : 1);
}
size_t weights_at(const pq_linear_desc* d) {
  return scales_at(d) + (static_cast<size_t>(d->M) * sizeof(float) + 15) / 16 * 16;
}

pq_status linear_codes(const void* q_dev, int32_t code_format, int64_t ldq, const float* s_x_dev, const int8_t* w_dev,
                       const float* s_w_dev, const float* bias_dev, int32_t* acc_dev, void* y_dev,
                       const pq_linear_desc* d, bool after_tokens, pq_stream_t stream) {
  if (!valid_linear(d)) return PQ_EINVAL;
  if (code_format != PQ_CODES_INT8 && code_format != PQ_CODES_F16) return PQ_EINVAL;
  if (d->M == 0) return PQ_OK;
  if (q_dev == nullptr || w_dev == nullptr || ldq < d->K || (acc_dev == nullptr && y_dev == nullptr)) return PQ_EINVAL;
  if (y_dev != nullptr && (s_x_dev == nullptr || s_w_dev == nullptr)) return PQ_EINVAL;
  if (!is_aligned(y_dev, bytes_of_type(d->y_type)) || !is_aligned(acc_dev, 4) || !is_aligned(s_x_dev, 4) ||
      !is_aligned(s_w_dev, 4) || !is_aligned(bias_dev, 4) || (code_format == PQ_CODES_F16 && !is_aligned(q_dev, 2)))
    return PQ_EINVAL;
  const size_t qe = code_format == PQ_CODES_F16 ? 2 : 1;
  const LinearArgs a = {q_dev,   ldq,   s_x_dev, w_dev,  d->ldw, s_w_dev, bias_dev,
                        acc_dev, y_dev, d->ldy,  d->M,   d->N,   d->K,    d->y_type,
                        is_aligned(q_dev, 16) && ldq * qe % 16 == 0};
  const bool wide = is_aligned(w_dev, 16) && d->ldw % 16 == 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (!(code_format == PQ_CODES_F16 && linear_tc_takes(a)) && d->M > 16ll * 65535)
    return PQ_EUNSUPPORTED;  // blocks along the grid's second axis
  if (code_format == PQ_CODES_F16 && linear_tc_takes(a))
    e = launch_linear_tc(a, after_tokens, s);
  else if (code_format == PQ_CODES_F16)
    e = wide ? launch_rows<true, true>(a, after_tokens, s) : launch_rows<true, false>(a, after_tokens, s);
  else if (wide && a.wide_q)
    e = d->M <= 8 ? launch_stream<1>(a, after_tokens, s) : launch_stream<2>(a, after_tokens, s);
  else
    e = wide ? launch_rows<false, true>(a, after_tokens, s) : launch_rows<false, false>(a, after_tokens, s);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

}  // namespace
}  // namespace pq

extern "C" {

pq_status palquant_quantize_tokens(const void* x_dev, int32_t x_type, int64_t ldx, int64_t M, int32_t K,
                                   int32_t code_format, void* q_dev, int64_t ldq, float* s_dev, pq_stream_t stream) {
  if (!pq::valid_type(x_type) || M < 0 || K < 1 || ldx < K || ldq < K) return PQ_EINVAL;
  if (code_format != PQ_CODES_INT8 && code_format != PQ_CODES_F16) return PQ_EINVAL;
  if (M == 0) return PQ_OK;
  if (M > pq::kMostTokens || K > 0x7FFFFFF8) return PQ_EUNSUPPORTED;  // blocks, and K rounded up to vectors of 8
  const bool half = code_format == PQ_CODES_F16;
  if (x_dev == nullptr || q_dev == nullptr || s_dev == nullptr || !pq::is_aligned(x_dev, pq::bytes_of_type(x_type)) ||
      !pq::is_aligned(q_dev, half ? 2 : 1) || !pq::is_aligned(s_dev, 4))
    return PQ_EINVAL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (x_type == PQ_F32)
    e = half ? pq::launch_tokens<float, true>(x_dev, ldx, M, K, q_dev, ldq, s_dev, s)
             : pq::launch_tokens<float, false>(x_dev, ldx, M, K, q_dev, ldq, s_dev, s);
  else if (x_type == PQ_F16)
    e = half ? pq::launch_tokens<__half, true>(x_dev, ldx, M, K, q_dev, ldq, s_dev, s)
             : pq::launch_tokens<__half, false>(x_dev, ldx, M, K, q_dev, ldq, s_dev, s);
  else
    e = half ? pq::launch_tokens<__nv_bfloat16, true>(x_dev, ldx, M, K, q_dev, ldq, s_dev, s)
             : pq::launch_tokens<__nv_bfloat16, false>(x_dev, ldx, M, K, q_dev, ldq, s_dev, s);
  return e == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

int32_t palquant_linear_code_format(const pq_linear_desc* d) {
  return pq::valid_linear(d) && d->M > 16 && pq::aligned_rows(d) ? PQ_CODES_F16 : PQ_CODES_INT8;
}

pq_status palquant_linear_i8(const void* q_dev, int32_t code_format, int64_t ldq, const float* s_x_dev,
                             const int8_t* w_dev, const float* s_w_dev, const float* bias_dev, int32_t* acc_dev,
                             void* y_dev, const pq_linear_desc* d, pq_stream_t stream) {
  return pq::linear_codes(q_dev, code_format, ldq, s_x_dev, w_dev, s_w_dev, bias_dev, acc_dev, y_dev, d, false, stream);
}

size_t palquant_linear_q8_scratch_bytes(const pq_linear_desc* d) {
  if (!pq::valid_linear(d) || d->M > pq::kMostTokens) return 0;
  if (!pq::copies_weights(d)) return pq::scales_at(d) + static_cast<size_t>(d->M) * sizeof(float);
  return pq::weights_at(d) + static_cast<size_t>(d->N) * static_cast<size_t>(pq::padded_k(d));
}

pq_status palquant_linear_q8(const void* x_dev, const int8_t* w_dev, const float* s_w_dev, const float* bias_dev,
                             void* y_dev, const pq_linear_desc* d, void* scratch_dev, size_t scratch_bytes,
                             pq_stream_t stream) {
  if (!pq::valid_linear(d)) return PQ_EINVAL;
  if (d->M == 0) return PQ_OK;
  if (d->M > pq::kMostTokens) return PQ_EUNSUPPORTED;
  if (x_dev == nullptr || w_dev == nullptr || s_w_dev == nullptr || y_dev == nullptr || scratch_dev == nullptr ||
      !pq::is_aligned(scratch_dev, 16) || scratch_bytes < palquant_linear_q8_scratch_bytes(d) ||
      !pq::is_aligned(y_dev, pq::bytes_of_type(d->y_type)) || !pq::is_aligned(s_w_dev, 4) ||
      !pq::is_aligned(bias_dev, 4))
    return PQ_EINVAL;
  const int32_t format = pq::q8_format(d);
  const int64_t pitch = pq::padded_k(d);
  char* scratch = static_cast<char*>(scratch_dev);
  float* s_x = reinterpret_cast<float*>(scratch + pq::scales_at(d));
  pq_linear_desc aligned = *d;
  if (pq::copies_weights(d)) {
    // before the tokens, so that the copy is complete when the product's first loads start
    int8_t* copy = reinterpret_cast<int8_t*>(scratch + pq::weights_at(d));
    const int64_t blocks = (d->N * (pitch / 16) + 255) / 256;
    pq::pq_align_weights<<<static_cast<unsigned>(blocks < 152 * 16 ? blocks : 152 * 16), 256, 0,
                           static_cast<cudaStream_t>(stream)>>>(w_dev, d->ldw, d->N, d->K, copy, pitch);
    if (cudaGetLastError() != cudaSuccess) return PQ_ECUDA;
    w_dev = copy;
    aligned.ldw = pitch;
  }
  const pq_status st = palquant_quantize_tokens(x_dev, d->x_type, d->ldx, d->M, d->K, format, scratch_dev, pitch, s_x, stream);
  if (st != PQ_OK) return st;
  return pq::linear_codes(scratch_dev, format, pitch, s_x, w_dev, s_w_dev, bias_dev, nullptr, y_dev, &aligned, true, stream);
}

}  // extern "C"
