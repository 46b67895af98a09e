// Attention over the paged 8-bit cache for few query rows (single tokens, short
// chunks; any other case, tile by tile).
//
// Mathematics.  With codes kc, vc and one scale for each page and head,
//   x_ij = scale log2(e) s_k(j) sum_d q_id kc_jd,   w_ij = 2^(x_ij + log2 s_v(j) - m_i),
//   o_id = sum_j w_ij vc_jd / sum_j w_ij / s_v(j),
// m_i the running maximum of x_ij + log2 s_v(j), up to a factor of 2^8 (2^2 for fp32).  Folding the value scale into the exponent keeps
// every w in the halves' range whatever the pages' scales are, so w can be a half value and the
// products with the codes run without a scale inside the MMA.  (A page whose value
// scale is 0 holds zeros only; it counts with kZeroPageScale.)
//
// Split.  Bound by the cache's bytes: each must be read once for all heads of a
// group.  A block takes one cache head, up to 16 query rows and a part of the token
// range; its 8 warps take 16-token steps in turn, each with a running maximum, sum
// and output of its own, joined through shared memory at the end.  Scores are computed
// transposed (tokens are the MMA's 16 rows, query rows its 8 columns: a group of up to
// 8 heads fills it), the probabilities turn into the second product's operand by
// an 8 x 8 transpose in registers, and the outputs are transposed too (16 rows of D).
// Codes come through shared memory, three or four steps of each warp in flight (16-byte
// asynchronous copies into a ring of the warp's own, no block-wide wait): with loads
// straight into registers a step waited for its page's id and then for its codes, and a
// batch of single tokens read 3.9 TB/s; now 5.5 (64 over up to 8192, 32 / 8 heads of 128: 122 us).  Of
// the rest, instructions (60 % of the issue slots, a third of them the codes' conversions) are one part and uneven shares
// were the other: 512 uncut (sequence, head) blocks of ragged lengths on 304 places keep 65 % of them at work as they come, the longest
// first 94 %, by a simulation of that schedule (143 us became 122).  Few query rows are spread over the chip by splitting
// the tokens; the parts' maxima, sums and outputs are joined by pq_kv8_join.
//
// Rounding.  Queries enter as halves scaled by a power of two for each row so that their largest
// element lies in [2^7, 2^8) (exact for 16-bit queries down to 2^-22 of it), w as
// halves (scaled, see kWShift); fp32 queries and their w carry a
// second half for the remainder (22 bits).  All sums are fp32.  exp2 and log2 are the chip's approximations
// (2^-22 or so of the result, for log2 of values near 1 absolute): below both.
#pragma once

#include <cuda_runtime.h>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_kv8.cuh"
#include "pq_tc.cuh"
#include "pq_tokens.cuh"

namespace pq {
namespace {

constexpr int kAttnWarps = 8;

// The block's share of the grid: the row tile changes fastest (its neighbours read
// the same codes).
struct Place {
  int tile, split, h, b;
};

__device__ __forceinline__ Place place_of(const AttnArgs& p) {
  Place r;
  unsigned i = blockIdx.x;
  if (p.cluster) {  // the parts of a row tile are one cluster
    r.split = i % p.splits;
    i /= p.splits;
    r.tile = i % p.row_tiles;
    i /= p.row_tiles;
    r.h = i % p.c.Hkv;
    r.b = i / p.c.Hkv;
    return r;
  }
  r.tile = i % p.row_tiles;
  i /= p.row_tiles;
  r.split = i % p.splits;
  i /= p.splits;
  r.h = i % p.c.Hkv;
  r.b = i / p.c.Hkv;
  return r;
}

__device__ __forceinline__ float log2_approx(float x) {
  float r;
  asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)) : "memory");
}
__device__ __forceinline__ uint4 lds_16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds_8(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
  return v;
}
// From a block of the cluster.
__device__ __forceinline__ float peer_f32(uint32_t addr, uint32_t rank) {
  uint32_t a;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float4 peer_f32x4(uint32_t addr, uint32_t rank) {
  uint32_t a;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float lds_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// A warp's ring: a step is 16 key rows and 16 value rows of DP bytes, then their scales.
__host__ __device__ constexpr int ring_steps(int DP) { return DP == 64 ? 4 : 3; }
__host__ __device__ constexpr int step_bytes(int DP) { return 32 * DP + 16; }
__host__ __device__ constexpr int ring_bytes(int DP) { return kAttnWarps * ring_steps(DP) * step_bytes(DP); }

// Where 16-byte piece c of a row lies: the pieces are exchanged so that the lanes that
// read together hit different banks.  Keys: rows g, pieces t; values: rows 2 t (and
// their odd neighbours), the pieces of D rows g.
template <int DP>
__device__ __forceinline__ uint32_t key_at(int row, int c) {
  return DP == 64 ? row * 64 + c * 16 : row * DP + ((c ^ ((row & 1) << 2)) << 4);
}
template <int DP>
__device__ __forceinline__ uint32_t value_at(int row, int c) {
  const int t = (row >> 1) & 3;
  if (DP == 64) return (row >> 1) * 128 + ((((row & 1) * 4 + c) ^ (t << 1)) << 4);
  if (DP == 128) return row * 128 + ((c ^ (t << 1)) << 4);
  return row * 256 + ((c ^ ((t & 1) | ((t >> 1) << 2))) << 4);
}

// DP: D rounded up to 64, 128 or 256; NT: tiles of 8 query rows; TWO: fp32 queries
// and outputs, each operand in two halves; VIEW: see AttnView.
template <typename T, int DP, int NT, bool TWO, int VIEW>
__global__ void __launch_bounds__(32 * kAttnWarps, DP <= 128 && NT == 1 && !TWO ? 2 : 1) pq_kv8_rows(const __grid_constant__ AttnArgs p) {
  constexpr int kC = DP / 64;        // 64-wide pieces of a key row
  constexpr int kJ = DP / 16;        // 16-row tiles of the transposed output
  constexpr int kRows = 8 * NT;
  constexpr int kHalves = TWO ? 2 : 1;                                  // of a query's element
  constexpr int kWHalves = TWO || kSecondHalf<T, VIEW> ? 2 : 1;         // of a weight
  constexpr float kGrowth = TWO ? kGrowF32 : kGrow, kShift = TWO ? kWShiftF32 : kWShift;
  constexpr int kSteps = ring_steps(DP);
  constexpr int kStep = step_bytes(DP);
  extern __shared__ __align__(16) uint8_t ring_raw[];
  __shared__ float row_factor[kRows];
  __shared__ float join_m[kAttnWarps][kRows], join_l[kAttnWarps][kRows];
  // the warps' outputs are joined in the ring's place
  static_assert(kAttnWarps / 2 * kJ * NT * 4 * 32 * 4 <= ring_bytes(DP), "join buffer");
  float (*join_o)[kJ * NT * 4][32] = reinterpret_cast<float (*)[kJ * NT * 4][32]>(ring_raw);
  Place w = place_of(p);
  if (p.in_order) w.b = longest_first(p, w.b, reinterpret_cast<int*>(ring_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int r0 = w.tile * kRows;
  const Span sp = span_of(p, w.b, r0, kRows);
  const int rows = sp.n * p.group;
  if (r0 >= rows) return;
  // (with sinks, steps are counted without the gap behind them; token() has it)
  const Walk walk = walk_of(p, sp);
  const int from = (VIEW == kSinks ? 0 : walk.gap) + w.split * p.chunk;
  const int end = VIEW == kSinks ? walk.end : sp.hi;
  const int to = min(end, from + p.chunk);
  const bool cluster = VIEW != kPlain && p.cluster;  // (a part without tokens takes part in the joining)
  if (w.split > 0 && from >= end && !cluster) return;
  auto token = [&](int s) { return VIEW == kSinks && s >= walk.head ? s + walk.gap : s; };
  const int D = p.c.D, C = D / 16;

  // ---- this warp's steps: tokens from + 16 (warp + 8 i) and up, kSteps - 1 of them ahead
  const int* table = p.a.page_table_dev + static_cast<int64_t>(w.b) * p.a.table_pitch;
  const uint32_t ring = smem_u32(ring_raw) + warp * kSteps * kStep;
  auto page_of = [&](int s) {  // page of a step's tokens
    const int slot = token(s) >> p.page_shift;
    return s < to && slot < p.a.table_pitch ? table[slot] : -1;
  };
  uint32_t valid = 0;  // bit i: the i-th step from now on that is in flight has a page
  auto issue = [&](int s, int id, int place, int ahead) {
    if (s < to) {
      if (id >= 0 && id < p.c.num_pages) {
        const int64_t ph = static_cast<int64_t>(id) * p.c.Hkv + w.h;
        const int64_t base = ((ph << p.page_shift) + (token(s) & (p.c.page_tokens - 1))) * D;
        const uint32_t at = ring + place * kStep;
        // 16 C pieces of each side; a token's pieces are neighbours
        const int8_t *k = p.c.k_dev + base + 16 * lane, *v = p.c.v_dev + base + 16 * lane;
        if (C == kJ) {
#pragma unroll
          for (int e = 0; e < DP; e += 32) {
            const int row = (e + lane) / kJ, c = lane % kJ;
            cp_async_16(at + key_at<DP>(row, c), k + 16 * e, 16);
            cp_async_16(at + 16 * DP + value_at<DP>(row, c), v + 16 * e, 16);
          }
        } else {
          for (int e = 0; e + lane < 16 * C; e += 32) {
            const int row = (e + lane) / C, c = e + lane - row * C;
            cp_async_16(at + key_at<DP>(row, c), k + 16 * e, 16);
            cp_async_16(at + 16 * DP + value_at<DP>(row, c), v + 16 * e, 16);
          }
        }
        if (lane == 0) cp_async_4(at + 32 * DP, p.c.k_scale_dev + ph);
        if (lane == 1) cp_async_4(at + 32 * DP + 4, p.c.v_scale_dev + ph);
        valid |= 1u << ahead;
      } else if (lane == 0) {
        atomicOr(p.err, PQ_ERR_PAGE);
      }
    }
    cp_async_commit();
  };
  const int s0 = from + 16 * warp;
  int next_id;
  {
    int ids[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) ids[i] = page_of(s0 + 16 * kAttnWarps * i);
#pragma unroll
    for (int i = 0; i < kSteps - 1; ++i) issue(s0 + 16 * kAttnWarps * i, ids[i], i, i);
    next_id = ids[kSteps - 1];
  }

  // ---- queries: row 8 j + g, columns 64 c + 16 t and up, as the MMA's second operand
  uint32_t qf[kHalves][NT][kC][8];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int r = r0 + 8 * j + g;
    const bool there = r < rows;
    const int64_t tok = p.a.cu_q_dev[w.b] + (there ? r / p.group : 0);
    const T* src = static_cast<const T*>(p.q) + tok * p.a.q_token_stride +
                   static_cast<int64_t>(w.h * p.group + (there ? r % p.group : 0)) * p.a.q_head_stride;
    Vec8<T> v[kC][2];
    uint32_t top = 0;
    // (the loads on their way at one time, not each behind a branch; rows past the end read the sequence's first and count as zeros)
    if (p.wide_q) {
#pragma unroll
      for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int d = 64 * c + 16 * t + 8 * i;
          v[c][i] = load8(src + (d < D ? d : 0), 8, true);
        }
#pragma unroll
      for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (!there || 64 * c + 16 * t + 8 * i >= D) v[c][i] = Vec8<T>{};
    } else {
#pragma unroll
      for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int d = 64 * c + 16 * t + 8 * i;
          v[c][i] = load8(src + d, there && d < D ? 8 : 0, false);
        }
    }
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) top = max(top, amax8(v[c][i]));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // 2^e <= largest magnitude < 2^(e+1); the row is scaled by 2^(7 - e)
    const int e = top >= 0x7F800000u ? 0 : max(static_cast<int>(top >> 23) - 127, -100);
    const float f = __int_as_float((127 + 7 - e) << 23);
    if (warp == 0 && t == 0) row_factor[8 * j + g] = p.a.scale * kLog2e * __int_as_float((127 - 7 + e) << 23);
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float a = to_f32(v[c][i].v[2 * k]) * f, b = to_f32(v[c][i].v[2 * k + 1]) * f;
          const uint32_t h = pack_half2(a, b);
          qf[0][j][c][4 * i + k] = h;
          if (TWO) {
            const __half2 hh = *reinterpret_cast<const __half2*>(&h);
            qf[kHalves - 1][j][c][4 * i + k] = pack_half2(a - __low2float(hh), b - __high2float(hh));
          }
        }
  }
  __syncthreads();
  // ---- this lane's score columns: rows 8 j + 2 t and 8 j + 2 t + 1
  float factor[NT][2];
  int lo[NT][2], hi[NT][2];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = r0 + 8 * j + 2 * t + i;
      factor[j][i] = row_factor[8 * j + 2 * t + i];
      const int at = sp.len - sp.n + r / p.group + 1;
      hi[j][i] = r >= rows ? 0 : p.a.causal ? min(at, sp.len) : sp.len;
      lo[j][i] = p.a.window > 0 ? max(0, at - p.a.window) : 0;
    }

  // tokens that every row of the tile sees
  int all_lo = 0, all_hi = sp.len;
  if (p.a.causal) {
    all_hi = max(0, sp.len - sp.n + r0 / p.group + 1);
    if (p.a.window > 0) all_lo = max(0, sp.len - sp.n + (min(rows, r0 + kRows) - 1) / p.group + 1 - p.a.window);
  }
  if (VIEW == kTree) all_hi = max(0, sp.len - sp.n);

  float m[NT][2], l[NT][2], o[kJ][NT][4];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) m[j][i] = kNone, l[j][i] = 0.0f;
#pragma unroll
  for (int i = 0; i < kJ; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][j][e] = 0.0f;

  int place = 0;
  for (int s = s0; s < to; s += 16 * kAttnWarps) {
    cp_async_wait<kSteps - 2>();
    __syncwarp();  // the step has arrived, and every lane is done with the one before
    const uint32_t at = ring + place * kStep;
    {
      const int ahead = s + 16 * kAttnWarps * (kSteps - 1);
      const int before = place == 0 ? kSteps - 1 : place - 1;
      issue(ahead, next_id, before, kSteps - 1);
      next_id = page_of(ahead + 16 * kAttnWarps);
      place = place + 1 == kSteps ? 0 : place + 1;
    }
    const bool there = valid & 1;
    valid >>= 1;
    if (!there) continue;
    // ---- codes: key rows g and g + 8
    uint4 kr[kC][2];
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        kr[c][i] = 64 * c + 16 * t < D ? lds_16(at + key_at<DP>(g + 8 * i, 4 * c + t)) : make_uint4(0, 0, 0, 0);
    const float sk = lds_f32(at + 32 * DP);
    const float sv0 = lds_f32(at + 32 * DP + 4);
    const float sv = sv0 == 0.0f ? kZeroPageScale : sv0;
    const float lv = log2_approx(sv), inv_v = exp2_approx(-lv);  // of one another, whatever the rounding

    // ---- scores
    float x[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[j][e] = 0.0f;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const uint32_t a[4] = {kr[c][0].x, kr[c][0].y, kr[c][0].z, kr[c][0].w};
      const uint32_t b[4] = {kr[c][1].x, kr[c][1].y, kr[c][1].z, kr[c][1].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t a0, a1, a2, a3;
        half_of_codes(a[i], a0, a2);
        half_of_codes(b[i], a1, a3);
#pragma unroll
        for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
          for (int j = 0; j < NT; ++j)
            mma_16x8x16(x[j], a0, a1, a2, a3, qf[hf][j][c][2 * i], qf[hf][j][c][2 * i + 1]);
      }
    }
    // ---- probabilities, of the running maximum as it was; only where a score has grown
    // past it by more than 2^8 (2^2 for fp32: w could leave the halves' range) is it brought up to date
    uint32_t pf[kWHalves][NT][2];
    float wv[NT][4], to_l[NT][2];
    bool grew = false;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        wv[j][e] = fmaf(x[j][e], sk * factor[j][e & 1], lv);
        to_l[j][e & 1] = inv_v;
      }
    const int s_tok = token(s);
    if ((s_tok < all_lo && !(VIEW == kSinks && s_tok + 16 <= p.sinks)) || s_tok + 16 > all_hi) {  // tokens that some row does not see
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int t0 = s_tok + g, t1 = t0 + 8;
          bool first_seen = t0 < hi[j][i] && (t0 >= lo[j][i] || (VIEW == kSinks && t0 < p.sinks));
          bool second_seen = t1 < hi[j][i] && (t1 >= lo[j][i] || (VIEW == kSinks && t1 < p.sinks));
          if (VIEW == kTree) {
            const int r = r0 + 8 * j + 2 * t + i;
            if (r < rows) {
              const uint32_t seen = drafts_seen(p.tree + (static_cast<int64_t>(p.a.cu_q_dev[w.b]) + r / p.group) * p.tree_pitch,
                                                p.tree_words, s_tok - (sp.len - sp.n));
              first_seen = first_seen && ((seen >> g) & 1u);
              second_seen = second_seen && ((seen >> (g + 8)) & 1u);
            }
          }
          if (!first_seen) wv[j][i] = kNone;
          if (!second_seen) wv[j][i + 2] = kNone;
          // a page that the row does not see adds nothing, even with a NaN scale
          if (!first_seen && !second_seen) to_l[j][i] = 0.0f;
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) grew |= wv[j][e] > m[j][e & 1] + kGrowth;
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        float alpha[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float top = fmaxf(m[j][i], fmaxf(wv[j][i], wv[j][i + 2]));
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
          alpha[i] = top == kNone ? 1.0f : exp2_approx(m[j][i] - top);
          m[j][i] = top;
          l[j][i] *= alpha[i];
        }
#pragma unroll
        for (int i = 0; i < kJ; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][j][e] *= alpha[e & 1];
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float base = m[j][e & 1] == kNone ? 0.0f : m[j][e & 1];
        wv[j][e] = exp2_approx(wv[j][e] - base + kShift);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) l[j][i] += (wv[j][i] + wv[j][i + 2]) * to_l[j][i];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t h = pack_half2(wv[j][2 * i], wv[j][2 * i + 1]);
        pf[0][j][i] = transpose_8x8(h);
        if (kWHalves == 2) {
          const __half2 hh = *reinterpret_cast<const __half2*>(&h);
          pf[kWHalves - 1][j][i] =
              transpose_8x8(pack_half2(wv[j][2 * i] - __low2float(hh), wv[j][2 * i + 1] - __high2float(hh)));
        }
      }
    }
    // ---- codes: value rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9
    uint32_t vr[4][DP / 32];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 2 * t + (i & 1) + 8 * (i >> 1);
      if (DP == 64) {
        const uint2 v = g * 8 < D ? lds_8(at + 16 * DP + value_at<DP>(row, g >> 1) + 8 * (g & 1)) : make_uint2(0, 0);
        vr[i][0] = v.x, vr[i][1] = v.y;
      } else {
#pragma unroll
        for (int c = 0; c < DP / 128; ++c) {
          const int piece = g * (DP / 128) + c;
          const uint4 v = piece < C ? lds_16(at + 16 * DP + value_at<DP>(row, piece)) : make_uint4(0, 0, 0, 0);
          vr[i][4 * c] = v.x, vr[i][4 * c + 1] = v.y, vr[i][4 * c + 2] = v.z, vr[i][4 * c + 3] = v.w;
        }
      }
    }
    // ---- outputs: tile i holds D rows g (DP/8) + 2 i (its rows 0-7) and + 2 i + 1 (rows 8-15)
#pragma unroll
    for (int c = 0; c < DP / 32; ++c) {
      uint32_t a01[4], a23[4];
      half_pairs_of_codes(vr[0][c], vr[1][c], a01);
      half_pairs_of_codes(vr[2][c], vr[3][c], a23);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int hf = 0; hf < kWHalves; ++hf)
#pragma unroll
          for (int j = 0; j < NT; ++j)
            mma_16x8x16(o[2 * c + i][j], a01[2 * i], a01[2 * i + 1], a23[2 * i], a23[2 * i + 1], pf[hf][j][0], pf[hf][j][1]);
    }
  }
  let_next_kernel_start();
  cp_async_wait<0>();
  __syncthreads();  // the ring is idle
  // ---- join the warps: sums over the lanes, then pairs of warps
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) l[j][i] += __shfl_xor_sync(0xffffffffu, l[j][i], d);
#pragma unroll
  for (int half = kAttnWarps / 2; half > 0; half >>= 1) {
    if (warp >= half && warp < 2 * half) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (g == 0) join_m[warp][8 * j + 2 * t + i] = m[j][i], join_l[warp][8 * j + 2 * t + i] = l[j][i];
#pragma unroll
        for (int i = 0; i < kJ; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) join_o[warp - half][(i * NT + j) * 4 + e][lane] = o[i][j][e];
      }
    }
    __syncthreads();
    if (warp < half) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        float mine[2], other[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float mo = join_m[warp + half][8 * j + 2 * t + i];
          const float top = fmaxf(m[j][i], mo), at = top == kNone ? 0.0f : top;
          mine[i] = exp2_approx(m[j][i] - at);
          other[i] = exp2_approx(mo - at);
          l[j][i] = l[j][i] * mine[i] + join_l[warp + half][8 * j + 2 * t + i] * other[i];
          m[j][i] = top;
        }
#pragma unroll
        for (int i = 0; i < kJ; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            o[i][j][e] = o[i][j][e] * mine[e & 1] + join_o[warp][(i * NT + j) * 4 + e][lane] * other[e & 1];
      }
    }
    __syncthreads();
  }
  if constexpr (VIEW != kPlain) {
    if (cluster) {
      // The parts' maxima, sums and outputs in every block's shared memory, joined in order: each block writes a share.
      float* mine_o = reinterpret_cast<float*>(ring_raw);
      if (warp == 0) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = 8 * j + 2 * t + i;
            if (g == 0) join_m[0][row] = m[j][i], join_l[0][row] = l[j][i];
#pragma unroll
            for (int k = 0; k < kJ; ++k)
              *reinterpret_cast<float2*>(mine_o + row * DP + g * (DP / 8) + 2 * k) = make_float2(o[k][j][i], o[k][j][i + 2]);
          }
      }
      cluster_sync();
      const uint32_t at_o = smem_u32(ring_raw), at_m = smem_u32(join_m[0]), at_l = smem_u32(join_l[0]);
      const int quads = D / 4, total = min(kRows, rows - r0) * quads;
      for (int e = w.split * (32 * kAttnWarps) + threadIdx.x; e < total; e += p.splits * (32 * kAttnWarps)) {
        const int row = e / quads, d = 4 * (e - row * quads);
        float top = kNone, pm[kMostCluster], pl[kMostCluster];
        float4 po[kMostCluster];
#pragma unroll
        for (int s = 0; s < kMostCluster; ++s)
          if (s < p.splits) {
            pm[s] = peer_f32(at_m + 4 * row, s);
            pl[s] = peer_f32(at_l + 4 * row, s);
            po[s] = peer_f32x4(at_o + 4 * (row * DP + d), s);
          }
#pragma unroll
        for (int s = 0; s < kMostCluster; ++s)
          if (s < p.splits) top = fmaxf(top, pm[s]);
        const float base = top == kNone ? 0.0f : top;
        float sum = 0.0f, y[4] = {};
#pragma unroll
        for (int s = 0; s < kMostCluster; ++s)
          if (s < p.splits) {
            const float f = exp2_approx(pm[s] - base);
            sum += pl[s] * f;
            y[0] += po[s].x * f, y[1] += po[s].y * f, y[2] += po[s].z * f, y[3] += po[s].w * f;
          }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int r = r0 + row, qi = r / p.group, hq = w.h * p.group + r % p.group;
        T* dst = static_cast<T*>(p.o) + (static_cast<int64_t>(p.a.cu_q_dev[w.b]) + qi) * p.a.o_token_stride +
                 static_cast<int64_t>(hq) * p.a.o_head_stride + d;
#pragma unroll
        for (int i = 0; i < 4; ++i) dst[i] = from_f32<T>(y[i] * inv);
      }
      cluster_sync();  // the others have read this block's part
      return;
    }
  }
  if (warp != 0) return;
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = r0 + 8 * j + 2 * t + i;
      if (r >= rows) continue;
      const int qi = r / p.group, hq = w.h * p.group + r % p.group;
      const int d0 = g * (DP / 8);
      if (p.splits > 1) {
        const int64_t at = ((static_cast<int64_t>(w.b) * p.a.max_q + qi) * p.a.Hq + hq) * p.splits + w.split;
        if (g == 0) p.ml[at] = make_float2(m[j][i], l[j][i]);
        float* dst = p.part + at * D + d0;
#pragma unroll
        for (int k = 0; k < kJ; ++k)
          if (d0 + 2 * k < D) *reinterpret_cast<float2*>(dst + 2 * k) = make_float2(o[k][j][i], o[k][j][i + 2]);
        continue;
      }
      const float inv = l[j][i] == 0.0f ? 0.0f : 1.0f / l[j][i];
      T* dst = static_cast<T*>(p.o) + (static_cast<int64_t>(p.a.cu_q_dev[w.b]) + qi) * p.a.o_token_stride +
               static_cast<int64_t>(hq) * p.a.o_head_stride + d0;
#pragma unroll
      for (int k = 0; k < kJ; k += 4) {
        Vec8<T> v;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          v.v[2 * u] = from_f32<T>(o[k + u][j][i] * inv);
          v.v[2 * u + 1] = from_f32<T>(o[k + u][j][i + 2] * inv);
        }
        if (d0 + 2 * k < D) store8(dst + 2 * k, v, 8, p.wide_o);
      }
    }
}

int padded_d(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

template <typename T, int DP, int NT, bool TWO, int VIEW>
cudaError_t launch_rows_as(const AttnArgs& p, unsigned grid, cudaStream_t s) {
  static int attr_set[64] = {0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !attr_set[dev]) {
    e = cudaFuncSetAttribute(pq_kv8_rows<T, DP, NT, TWO, VIEW>, cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes(DP));
    if (e != cudaSuccess) return e;
    if (dev < 64) attr_set[dev] = 1;
  }
  if (VIEW != kPlain && p.cluster) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(32 * kAttnWarps);
    cfg.dynamicSmemBytes = ring_bytes(DP);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(p.splits);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, pq_kv8_rows<T, DP, NT, TWO, VIEW>, p);
  }
  pq_kv8_rows<T, DP, NT, TWO, VIEW><<<grid, 32 * kAttnWarps, ring_bytes(DP), s>>>(p);
  return cudaGetLastError();
}

template <typename T, bool TWO, int VIEW>
cudaError_t launch_rows(const AttnArgs& p, unsigned grid, int nt, cudaStream_t s) {
  const int dp = padded_d(p.c.D);
  if (dp == 64) return nt == 1 ? launch_rows_as<T, 64, 1, TWO, VIEW>(p, grid, s) : launch_rows_as<T, 64, 2, TWO, VIEW>(p, grid, s);
  if (dp == 128) return nt == 1 ? launch_rows_as<T, 128, 1, TWO, VIEW>(p, grid, s) : launch_rows_as<T, 128, 2, TWO, VIEW>(p, grid, s);
  return launch_rows_as<T, 256, 1, TWO, VIEW>(p, grid, s);
}

}  // namespace

template <int VIEW>
cudaError_t launch_attn_rows(const AttnArgs& p, unsigned grid, int nt, cudaStream_t s) {
  if (p.a.type == PQ_F32) return launch_rows<float, true, VIEW>(p, grid, nt, s);
  if (p.a.type == PQ_F16) return launch_rows<__half, false, VIEW>(p, grid, nt, s);
  return launch_rows<__nv_bfloat16, false, VIEW>(p, grid, nt, s);
}

}  // namespace pq
