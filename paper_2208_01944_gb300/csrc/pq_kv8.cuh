// What the attention kernels over the 8-bit cache share.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "palquant.h"
#include "pq_tokens.cuh"

namespace pq {

struct AttnArgs {
  pq_kv8_cache c;
  pq_kv8_attn a;
  const void* q;
  void* o;
  int group;       // query heads of one cache head
  int page_shift;  // log2(page_tokens)
  int row_tiles;   // tiles of query rows (query, head of the group) of one cache head
  int splits;      // parts of the token range, joined by a second kernel if more than one
  int chunk;       // tokens of one part, a multiple of 128
  int align;       // the first part of a row tile begins at a multiple of this
  float2* ml;      // [B * max_q * Hq][splits]: running maximum and sum of every part
  float* part;     // [B * max_q * Hq][splits][D]: its unnormalised output
  unsigned int* err;
  uint64_t wait_limit_ns;
  bool wide_q, wide_o;  // rows on 16-byte boundaries
};

bool valid_kv8_cache(const pq_kv8_cache* c);

// Tiles of 256 query rows on the tensor cores; fp32 queries and D above 128 are not its.
bool attn_tc_takes(const pq_kv8_cache& c, const pq_kv8_attn& a);
constexpr int kAttnTcRows = 256;
constexpr int kAttnTcTokens = 128;
cudaError_t launch_attn_tc(const AttnArgs& p, unsigned grid, cudaStream_t stream);

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -INFINITY;

// The value scale that a page of zero values (scale 0) counts with.  Its weights 2^(x + log2 s_v) add
// nothing to the outputs, only to the sum, where s_v is divided out again; but they take part in the running
// maximum, and whatever lies below 2^-30 of that is lost to the outputs.  So it has to lie below every
// other page's (2^-40 and up), and within 2^100 of the largest (2^40), for the sum's own terms to stay in fp32's range.
constexpr float kZeroPageScale = 0x1p-60f;

// log2 by which a maximum may grow before the sums and outputs are rescaled, and by which
// the weights are scaled before they become halves: those of the running maximum are 2^6, the
// largest below 2^14, and a weight keeps a half's full 11 bits down to 2^-20 of the maximum (2^-14 if it were not
// scaled).  fp32 carries the rest of a weight in a second half, which wants more room
// below: 22 bits down to 2^-16 of the maximum (2^-9 with the others' scaling), and a maximum that may grow by 2^2.
constexpr float kGrow = 8.0f, kWShift = 6.0f;
constexpr float kGrowF32 = 2.0f, kWShiftF32 = 13.0f;

// (within 2^-22 of the result; a weight is rounded to 11 bits next, or to twice 11 for fp32)
__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Tokens that the query rows [r0, r0 + rows) of sequence b may see: [lo, hi).
struct Span {
  int n, len;  // queries and tokens of the sequence
  int lo, hi;
};

__device__ __forceinline__ Span span_of(const AttnArgs& p, int b, int r0, int rows) {
  Span s;
  s.n = min(p.a.cu_q_dev[b + 1] - p.a.cu_q_dev[b], p.a.max_q);
  s.len = max(0, min(p.a.len_dev[b], p.a.max_len));
  s.lo = 0;
  s.hi = s.len;
  if (p.a.causal) {
    const int last = min(s.n * p.group, r0 + rows) - 1;
    s.hi = min(s.len, s.len - s.n + last / p.group + 1);
    if (p.a.window > 0) s.lo = max(0, s.len - s.n + r0 / p.group + 1 - p.a.window);
  }
  return s;
}

}  // namespace pq
