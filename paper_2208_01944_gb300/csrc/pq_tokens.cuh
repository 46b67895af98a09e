// Device-side building blocks of the 8-bit transformer kernels: element types,
// signed 8-bit codes and their half values, the warp-level half-precision MMA.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cfloat>
#include <cstdint>

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
    uint4* q = reinterpret_cast<uint4*>(&r);
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(r) / 16); ++i) q[i] = reinterpret_cast<const uint4*>(p)[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = i < n ? p[i] : from_f32<T>(0.0f);
  }
  return r;
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const Vec8<T>& r, int n, bool wide) {
  if (wide) {
    const uint4* q = reinterpret_cast<const uint4*>(&r);
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

template <typename T>
__device__ __forceinline__ uint32_t amax8(const Vec8<T>& r) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, abs_bits(to_f32(r.v[i])));
  return m;
}

__device__ __forceinline__ float scale_of_amax(uint32_t bits) {
  if (bits >= 0x7F800000u) return __int_as_float(0x7FC00000);  // NaN
  const float s = __fmul_rn(__uint_as_float(bits), kInv127);
  return s < FLT_MIN ? 0.0f : s;
}

// fl(1/s), 0 for the scales 0 and NaN (whose codes are 0).
__device__ __forceinline__ float inverse_of_scale(float s) { return s > 0.0f ? __frcp_rn(s) : 0.0f; }

// clamp(rint(fl(x * inv)), -127, 127); 0 where inv is 0, whatever x is.
__device__ __forceinline__ int code_of(float x, float inv) {
  const int c = __float2int_rn(__fmul_rn(x, inv));  // NaN (an infinity or NaN under inv = 0) -> 0
  return min(max(c, -127), 127);
}

__device__ __forceinline__ uint32_t pack_bytes(int a, int b, int c, int d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

template <typename T>
__device__ __forceinline__ uint2 codes8(const Vec8<T>& r, float inv) {
  int c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = code_of(to_f32(r.v[i]), inv);
  return make_uint2(pack_bytes(c[0], c[1], c[2], c[3]), pack_bytes(c[4], c[5], c[6], c[7]));
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
