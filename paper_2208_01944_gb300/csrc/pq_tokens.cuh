// Device-side building blocks of the 8-bit transformer kernels: element types,
// signed 8-bit codes and their half values, the warp-level half-precision MMA.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cfloat>
#include <cstdint>
#include <cstring>

#include "pq_device.cuh"

namespace pq {

constexpr float kInv127 = 1.0f / 127.0f;

// ---------------------------------------------------------------- elements
template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Eight consecutive elements in registers as they lie in memory.
template <typename T>
struct alignas(16) Vec8 {
  T v[8];
};

// n of eight elements (the others zero); `wide`: all eight are there and the
// address is 16-byte aligned.
template <typename T>
__device__ __forceinline__ Vec8<T> load8(const T* p, int n, bool wide) {
  Vec8<T> r;
  if (wide) {
    uint4 q[sizeof(r) / 16];
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(r) / 16); ++i) q[i] = reinterpret_cast<const uint4*>(p)[i];
    memcpy(&r, q, sizeof(r));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = i < n ? p[i] : from_f32<T>(0.0f);
  }
  return r;
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const Vec8<T>& r, int n, bool wide) {
  if (wide) {
    uint4 q[sizeof(r) / 16];
    memcpy(q, &r, sizeof(r));
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(r) / 16); ++i) reinterpret_cast<uint4*>(p)[i] = q[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = r.v[i];
  }
}

// ------------------------------------------------------------------ scales
// The largest magnitude is kept as the bits of |x|: their order as integers is
// that of the values, with infinities and NaN above every number.
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Of eight elements, as 32-bit float bits.  16-bit elements are compared in pairs.
template <typename T>
__device__ __forceinline__ uint32_t amax8(const Vec8<T>& r) {
  if constexpr (sizeof(T) == 2) {
    uint32_t w[4];
    memcpy(w, &r, sizeof(w));
    uint32_t m = __vmaxu2(__vmaxu2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu), __vmaxu2(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
    m = max(m & 0xFFFFu, m >> 16);
    const unsigned short bits = static_cast<unsigned short>(m);
    T top;
    memcpy(&top, &bits, sizeof(top));
    return abs_bits(to_f32(top));
  } else {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, abs_bits(to_f32(r.v[i])));
    return m;
  }
}

__device__ __forceinline__ float scale_of_amax(uint32_t bits) {
  if (bits >= 0x7F800000u) return __int_as_float(0x7FC00000);  // NaN
  const float s = __fmul_rn(__uint_as_float(bits), kInv127);
  return s < FLT_MIN ? 0.0f : s;
}

// fl(1/s), 0 for the scales 0 and NaN (whose codes are 0).
__device__ __forceinline__ float inverse_of_scale(float s) { return s > 0.0f ? __frcp_rn(s) : 0.0f; }

// clamp(rint(fl(x * inv)), -127, 127) of values that lie under the scale: fl(x * inv) is
// at most 127 (1 + 2^-22) and needs no clamp, and adding 1.5 * 2^23 rounds it to the nearest
// integer, half to even, into the low bits of the sum (a conversion to an integer runs at
// a quarter of the rate of an addition's half).  Where inv is 0 the codes are 0
// whatever x is.
constexpr float kRound = 12582912.0f;  // 1.5 * 2^23
__device__ __forceinline__ float rounded_bits(float x, float inv) { return __fadd_rn(__fmul_rn(x, inv), kRound); }

// (a, b) as rounded_bits.  Not with the packed forms of both operations: the compiler
// contracts a packed product and sum into one rounding, which decides ties differently.
__device__ __forceinline__ void rounded_pair(float a, float b, float inv, float& x, float& y) {
  x = rounded_bits(a, inv);
  y = rounded_bits(b, inv);
}

__device__ __forceinline__ uint32_t low_bytes(float a, float b, float c, float d) {
  return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040),
                     __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
}

template <typename T>
__device__ __forceinline__ uint2 codes8(const Vec8<T>& r, float inv) {
  float c[8];
#pragma unroll
  for (int i = 0; i < 8; i += 2) rounded_pair(to_f32(r.v[i]), to_f32(r.v[i + 1]), inv, c[i], c[i + 1]);
  const uint2 w = make_uint2(low_bytes(c[0], c[1], c[2], c[3]), low_bytes(c[4], c[5], c[6], c[7]));
  return inv > 0.0f ? w : make_uint2(0, 0);
}

// The same codes as halves.
template <typename T>
__device__ __forceinline__ Vec8<__half> half_codes8(const Vec8<T>& r, float inv) {
  Vec8<__half> h;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float a, b;
    rounded_pair(to_f32(r.v[i]), to_f32(r.v[i + 1]), inv, a, b);
    add2_rn(a, b, -kRound, a, b);
    uint32_t v;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(b), "f"(a));
    w[i / 2] = inv > 0.0f ? v : 0u;
  }
  memcpy(&h, w, sizeof(w));
  return h;
}

// Four codes as fp32: the byte u = code + 128 in the low bits of 2^23 + u, less 2^23 + 128.
__device__ __forceinline__ void floats_of_codes(uint32_t w, float (&r)[4]) {
  const uint32_t u = w ^ 0x80808080u;
  add2_rn(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440)), __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7441)), -8388736.0f,
          r[0], r[1]);
  add2_rn(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7442)), __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7443)), -8388736.0f,
          r[2], r[3]);
}

// Largest of all threads' values, for blocks of up to 8 warps; red: 8 words of
// shared memory.  Every thread of the block calls it.
__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t* red) {
  m = __reduce_max_sync(0xffffffffu, m);
  const int warp = threadIdx.x >> 5, nw = (blockDim.x + 31) >> 5;
  if ((threadIdx.x & 31) == 0) red[warp] = m;
  __syncthreads();
  for (int w = 0; w < nw; ++w) m = max(m, red[w]);
  return m;
}

// ------------------------------------------------------ codes as half values
// A signed byte c, its top bit flipped, is u = c + 128 in [0, 255]; the half
// with bits 0x6400 | u is 1024 + u, and subtracting 1152 leaves c exactly.
// Four codes cost one exclusive or, two byte permutes and two packed subtractions.
__device__ __forceinline__ uint32_t sub_half2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

__device__ __forceinline__ void half_of_codes(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const uint32_t u = w ^ 0x80808080u;
  lo = sub_half2(__byte_perm(u, 0x64646464u, 0x4140), 0x64806480u);
  hi = sub_half2(__byte_perm(u, 0x64646464u, 0x4342), 0x64806480u);
}

// Codes of two rows (a, b) at four columns as pairs (a, b) of halves, a column each.
__device__ __forceinline__ void half_pairs_of_codes(uint32_t a, uint32_t b, uint32_t (&r)[4]) {
  const uint32_t lo = __byte_perm(a, b, 0x5140) ^ 0x80808080u;  // a0 b0 a1 b1
  const uint32_t hi = __byte_perm(a, b, 0x7362) ^ 0x80808080u;  // a2 b2 a3 b3
  r[0] = sub_half2(__byte_perm(lo, 0x64646464u, 0x4140), 0x64806480u);
  r[1] = sub_half2(__byte_perm(lo, 0x64646464u, 0x4342), 0x64806480u);
  r[2] = sub_half2(__byte_perm(hi, 0x64646464u, 0x4140), 0x64806480u);
  r[3] = sub_half2(__byte_perm(hi, 0x64646464u, 0x4342), 0x64806480u);
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// d += a b, one warp: a 16 x 16 (row-major halves), b 16 x 8 (column-major), fp32 sums.
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                            uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Transpose of an 8 x 8 matrix of halves held one row per four lanes.
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

// ------------------------------------------------- tensor memory and operands
// K-major operand in the 128-byte swizzle: rows of 128 bytes, groups of 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t sw128_desc(uint32_t addr) {
  return static_cast<uint64_t>((addr >> 4) & 0x3FFFu) | (static_cast<uint64_t>(1) << 16) |
         (static_cast<uint64_t>(1024 >> 4) << 32) | (static_cast<uint64_t>(1) << 46) | (static_cast<uint64_t>(2) << 61);
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

// A launch that is a programmatic dependent of the kernel before it waits here
// until that kernel's results are visible.
__device__ __forceinline__ void wait_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

inline size_t bytes_of_type(int32_t t) { return t == 0 ? 4 : 2; }
inline bool is_aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace pq
