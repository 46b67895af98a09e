// What the attention kernels over the 8-bit cache share.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

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
  bool cluster;         // a row tile's parts are a cluster of blocks, which join them: no scratch, no second kernel
  bool in_order;        // sequences are taken the longest first
  int sinks;            // kSinks: first tokens that stay visible (0 in the other views)
  const uint32_t* tree; // kTree: which drafts each draft sees, tree_words words a row
  int64_t tree_pitch;
  int tree_words;
};

// What a query sees: the tokens up to it (all of them, or through a window) or every token; through
// a window with the first tokens; the text before the drafts and the drafts that its bits name.
enum AttnView : int { kPlain = 0, kSinks = 1, kTree = 2 };

// With half-precision outputs an 11-bit weight is off by as much as the output's own rounding: together sqrt(2) of
// it (measured against 64 bits: 3.1e-4 of the outputs' norm, the rounding alone 2.0e-4).  The views with sinks and drafts carry the
// rest of a weight in a second half there, as fp32 does.  bfloat16's own rounding is 1.7e-3 of the norm: 11-bit weights add at most 1 % to it, and
// a second half would cost what it costs halves (us, bfloat16 / half: 2 prompts of 4096 through a window 284 / 354, 32 users' two dozen
// drafts 86 / 99).
template <typename T, int VIEW>
constexpr bool kSecondHalf = VIEW != kPlain && sizeof(T) == 2 && !std::is_same<T, __nv_bfloat16>::value;

constexpr int kMostCluster = 8;

bool valid_kv8_cache(const pq_kv8_cache* c);

// Few query rows of a cache head, any type and D: nt tiles of 8 a block.
template <int VIEW>
cudaError_t launch_attn_rows(const AttnArgs& p, unsigned grid, int nt, cudaStream_t stream);

// Tiles of 256 query rows on the tensor cores; fp32 queries and D above 128 are not its.
bool attn_tc_takes(const pq_kv8_cache& c, const pq_kv8_attn& a);
constexpr int kAttnTcRows = 256;
constexpr int kAttnTcTokens = 128;
template <int VIEW>
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

// The i-th sequence, the longest first (of equals the first; those without queries last).  Every thread of a block of 256 or
// more calls; `room`, B + 1 numbers of shared memory, is free again afterwards.  Up to 8 neighbours count for one sequence.
constexpr int kMostInOrder = 128;
__device__ __forceinline__ int longest_first(const AttnArgs& p, int i, int* room) {
  const int B = p.a.B, shift = B <= 32 ? 3 : B <= 64 ? 2 : 1;
  const int b = threadIdx.x >> shift, part = threadIdx.x & ((1 << shift) - 1);
  int mine = -1;
  if (b < B && p.a.cu_q_dev[b + 1] > p.a.cu_q_dev[b]) mine = max(0, p.a.len_dev[b]);
  if (b < B && part == 0) room[b] = mine;
  __syncthreads();
  int before = 0;
  if (b < B) {
#pragma unroll 4
    for (int j = part; j < B; j += 1 << shift) {
      const int other = room[j];
      before += other > mine || (other == mine && j < b);
    }
  }
  for (int k = 1; k < 1 << shift; k *= 2) before += __shfl_xor_sync(0xffffffffu, before, k);
  if (b < B && part == 0 && before == i) room[B] = b;
  __syncthreads();
  const int r = room[B];
  __syncthreads();
  return r;
}

// How a row tile walks through its tokens: steps of 16 or 128 (the kernel's `align`) through the first
// `head` of them, then from `head` + gap on, `end` in all.  The head holds the sinks that lie before the
// span; it and the gap are multiples of a step, so no step lies on both sides.
struct Walk {
  int head, gap, end;
};

__device__ __forceinline__ Walk walk_of(const AttnArgs& p, const Span& s) {
  const int first = s.lo & ~(p.align - 1);
  Walk w;
  w.head = min((p.sinks + p.align - 1) & ~(p.align - 1), first);
  w.gap = first - w.head;
  w.end = s.hi - w.gap;
  return w;
}

// The lowest n of 32 bits (none below 0, all from 32 on).
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 32 ? 0xFFFFFFFFu : (1u << max(n, 0)) - 1u; }

// Which of the drafts off to off + 31 a draft sees, from the `words` words of its row; what lies
// before draft 0 is the text, which it sees.
__device__ __forceinline__ uint32_t drafts_seen(const uint32_t* row, int words, int off) {
  if (off <= -32) return 0xFFFFFFFFu;
  if (off < 0) return (row[0] << -off) | first_bits(-off);
  const int w = off >> 5;
  return __funnelshift_r(w < words ? row[w] : 0u, w + 1 < words ? row[w + 1] : 0u, off & 31);
}

}  // namespace pq
