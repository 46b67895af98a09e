// Attention over the paged 8-bit cache: what a call checks, which kernel it takes (pq_kv8_rows for few query
// rows of a cache head, pq_kv8_tiles for many), how the token range is cut, and the kernel that joins its parts.
#include <cuda_runtime.h>

#include <algorithm>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_kv8.cuh"
#include "pq_tokens.cuh"

namespace pq {
namespace {

// Joins the parts of one query row: W warps each, which take the parts in turn (one
// warp would wait for hundreds of them one after the other).
template <typename T, int W>
__global__ void __launch_bounds__(256) pq_kv8_join(const __grid_constant__ AttnArgs p, int tile_rows) {
  __shared__ float sums[W > 1 ? 8 : 1][W > 1 ? 260 : 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % W;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * (8 / W) + warp / W;
  const int hq = static_cast<int>(at % p.a.Hq);
  const int64_t rest = at / p.a.Hq;
  const int qi = static_cast<int>(rest % p.a.max_q);
  const int64_t b = rest / p.a.max_q;
  wait_previous_kernel();
  const bool row = b < p.a.B;
  const int r = qi * p.group + hq % p.group;
  Span sp = {};
  if (row) sp = span_of(p, static_cast<int>(b), r / tile_rows * tile_rows, tile_rows);
  // the parts that the row's tile was cut into (at least the first is there)
  const Walk walk = walk_of(p, sp);
  const int parts = row && qi < sp.n ? max(1, min(p.splits, (walk.end + p.chunk - 1) / p.chunk)) : 0;
  const float2* ml = p.ml + at * p.splits;
  float top = kNone;
  for (int s = lane; s < parts; s += 32) top = fmaxf(top, ml[s].x);
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  const float base = top == kNone ? 0.0f : top;
  float l = 0.0f, o[8] = {};
#pragma unroll 4
  for (int s = part; s < parts; s += W) {
    const float2 v = ml[s];
    const float f = exp2_approx(v.x - base);
    l += v.y * f;
    const float* src = p.part + (at * p.splits + s) * p.c.D;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (lane + 32 * k < p.c.D) o[k] += src[lane + 32 * k] * f;
  }
  if (W > 1) {
#pragma unroll
    for (int k = 0; k < 8; ++k) sums[W > 1 ? warp : 0][W > 1 ? lane + 32 * k : 0] = o[k];
    if (lane == 0) sums[W > 1 ? warp : 0][W > 1 ? 256 : 0] = l;
    __syncthreads();
    if (part != 0) return;
    for (int i = 1; i < W; ++i) {
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] += sums[W > 1 ? warp + i : 0][W > 1 ? lane + 32 * k : 0];
      l += sums[W > 1 ? warp + i : 0][W > 1 ? 256 : 0];
    }
  }
  if (parts == 0) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  T* dst = static_cast<T*>(p.o) + (static_cast<int64_t>(p.a.cu_q_dev[b]) + qi) * p.a.o_token_stride +
           static_cast<int64_t>(hq) * p.a.o_head_stride;
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (lane + 32 * k < p.c.D) dst[lane + 32 * k] = from_f32<T>(o[k] * inv);
}

// ---------------------------------------------------------------------- host
int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    sms = 0;
  return sms > 0 ? sms : 152;
}

// Tiles of 8 query rows of one block: two where there are more than 8 rows and the
// outputs of 16 fit the registers.
int row_tiles_of_block(const pq_kv8_cache* c, const pq_kv8_attn* a) {
  const int64_t rows = static_cast<int64_t>(a->max_q) * (a->Hq / c->Hkv);
  return rows <= 8 || c->D > 128 ? 1 : 2;
}

bool valid_attn(const pq_kv8_cache* c, const pq_kv8_attn* a) {
  if (!valid_kv8_cache(c) || a == nullptr) return false;
  if (a->type != PQ_F32 && a->type != PQ_F16 && a->type != PQ_BF16) return false;
  if (a->B < 0 || a->max_q < 0 || a->max_len < 0 || a->table_pitch < 0 || a->window < 0) return false;
  if (a->Hq < 1 || a->Hq % c->Hkv != 0 || a->Hq / c->Hkv > 64) return false;
  if ((a->causal != 0 && a->causal != 1) || (a->causal == 0 && a->window != 0)) return false;
  if (a->q_token_stride < 0 || a->q_head_stride < 0 || a->o_token_stride < 0 || a->o_head_stride < 0) return false;
  return !(a->scale != a->scale);
}

// Query rows, and with them tiles and blocks before the tokens are cut, are counted in 32 bits.
// (The product of three 32-bit numbers may pass 64 bits; as doubles it is exact far beyond the limit.)
// Positions are too, and a part's end or a warp's next step lies up to a part beyond the last: up to 2^30 of them.
bool countable(const pq_kv8_attn* a) {
  return a->max_len <= 1 << 30 && a->max_q <= 1 << 30 && static_cast<double>(a->B) * a->max_q * a->Hq <= static_cast<double>(0x7FFFFFFF);
}

// The call with a window that no text is longer than taken as none: the same result, and the kernels'
// position - window stays in 32 bits where queries outnumber the tokens (positions below 0).
pq_kv8_attn without_idle_window(const pq_kv8_attn* a) {
  pq_kv8_attn r = *a;
  if (r.window >= r.max_len) r.window = 0;
  return r;
}

// Which kernel, its row tiles, and the parts of the token range.  Few query rows are
// spread over the chip by cutting the tokens: two blocks an SM (as many as fit) of at
// least 256 tokens (two steps of every warp), or, on the tensor cores, one block an SM of
// at least 512.  Four blocks an SM cost the joining kernel more than they won (one token
// over 130001: 46 us, two 38 us).
struct Plan {
  bool tc;
  int rows;  // query rows of a tile
};

//
// The views with sinks and drafts (`fine`) go further where little is to be done (us in a graph): a range of up to 512 tokens stays in
// one part, without the joining kernel (one token through a window of 256: 5.8, two parts 7.3); and where parts of 128 tokens find room
// on the chip at one time, the rows kernel takes them, more than 40 rows too (12 drafts x 4 heads over 2000: 9.9, parts of 256 11.8; on
// the tensor cores parts of 128 10.7, of 512 15.1).  Up to 8 parts of at most 512 tokens are the blocks of a cluster, which join them
// themselves (the same drafts 9.2).  Plain attention keeps the parts, and with them the bits, that it always had.
Plan plan_attention(const pq_kv8_cache* c, const pq_kv8_attn* a, AttnArgs* p, bool fine) {
  Plan plan;
  plan.tc = attn_tc_takes(*c, *a);
  plan.rows = plan.tc ? kAttnTcRows : 8 * row_tiles_of_block(c, a);
  const int64_t head16 = (static_cast<int64_t>(p->sinks) + 15) / 16 * 16;
  const int64_t tokens = a->window > 0 ? std::min<int64_t>(a->max_len, head16 + a->window + a->max_q + 16) : a->max_len;
  const int64_t small_rows = 8 * row_tiles_of_block(c, a);
  const int64_t small_units = static_cast<int64_t>(a->B) * c->Hkv * ((static_cast<int64_t>(a->max_q) * (a->Hq / c->Hkv) + small_rows - 1) / small_rows);
  const bool roomy = fine && small_units <= 2 * sm_count() && small_units * ((tokens + 127) / 128) <= 2 * sm_count();
  if (roomy) {
    plan.tc = false;
    plan.rows = static_cast<int>(small_rows);
  }
  p->align = plan.tc ? kAttnTcTokens : 16;
  p->row_tiles = static_cast<int>((static_cast<int64_t>(a->max_q) * (a->Hq / c->Hkv) + plan.rows - 1) / plan.rows);
  // tokens that one row tile can see, from a multiple of `align` on
  int64_t range = a->max_len;
  const int64_t head = (static_cast<int64_t>(p->sinks) + p->align - 1) / p->align * p->align;
  if (a->window > 0) range = std::min<int64_t>(range, head + a->window + plan.rows + p->align);
  range = std::max<int64_t>(range, 1);
  const int64_t units = static_cast<int64_t>(a->B) * c->Hkv * p->row_tiles;
  const int64_t want = ((plan.tc ? 1 : 2) * static_cast<int64_t>(sm_count()) + units - 1) / units;
  const int64_t least = fine && !plan.tc && range <= 512 ? 512 : plan.tc ? 512 : roomy ? 128 : 256;
  const int64_t splits = std::max<int64_t>(1, std::min(want, (range + least - 1) / least));
  const int64_t chunk = ((range + splits - 1) / splits + 127) / 128 * 128;
  p->chunk = static_cast<int>(std::min<int64_t>(chunk, 0x7FFFFF80));
  p->splits = static_cast<int>((range + chunk - 1) / chunk);
  if (roomy && range > 512 && range <= 512 * kMostCluster) {
    p->chunk = static_cast<int>(((range + kMostCluster - 1) / kMostCluster + 127) / 128 * 128);
    p->splits = static_cast<int>((range + p->chunk - 1) / p->chunk);
    p->cluster = p->splits > 1;
  }
  return plan;
}

// Blocks start in order, and whichever comes last keeps the call: so where there are up to four times as many as run at one time, they
// take the longest texts first.  It costs each block a look at all lengths, which short texts, many sequences and many rounds do
// not pay back.  Single tokens, 32 / 8 heads of 128, us in order / as they come: 64 over 2048 to 8192 117 / 144, 128 over 64 to 4000
// 66 / 81 (4 cached heads), 64 over 64 to 1024 26.5 / 26.5, and of one length 64 over 8192 191 / 189, over 1024 37 / 36; 512 over 256
// 52 / 16 (one cached head).
// Through a window, lengths say little.  Results do not depend on it.
bool in_order(const pq_kv8_attn& a, const Plan& plan, unsigned grid) {
  const unsigned places = static_cast<unsigned>((plan.tc ? 1 : 2) * sm_count());
  return a.window == 0 && a.max_len >= 2048 && a.B > 1 && a.B <= kMostInOrder && grid > places && grid <= 4 * places;
}

template <typename T>
cudaError_t launch_join(const AttnArgs& p, int tile_rows, cudaStream_t s) {
  const int64_t rows = static_cast<int64_t>(p.a.B) * p.a.max_q * p.a.Hq;
  cudaLaunchConfig_t cfg = {};
  const bool many = p.splits > 8;
  cfg.gridDim = dim3(static_cast<unsigned>(many ? rows : (rows + 7) / 8));
  cfg.blockDim = dim3(256);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return many ? cudaLaunchKernelEx(&cfg, pq_kv8_join<T, 8>, p, tile_rows) : cudaLaunchKernelEx(&cfg, pq_kv8_join<T, 1>, p, tile_rows);
}

size_t scratch_of(const AttnArgs& p) {
  if (p.splits <= 1 || p.cluster) return 0;
  const size_t parts = static_cast<size_t>(p.a.B) * p.a.max_q * p.a.Hq * p.splits;
  return parts * sizeof(float2) + parts * p.c.D * sizeof(float);
}

// What a call sees, beside its descriptor.
struct View {
  AttnView kind;
  int32_t sinks;
  const pq_kv8_tree* tree;
};

// Sinks beside a causal view; drafts beside a causal one without a window, with enough bits for each.
bool valid_view(const pq_kv8_attn* a, const View& v) {
  if (v.kind == kSinks) return a->causal == 1 && v.sinks >= 0;
  if (v.kind == kTree)
    return a->causal == 1 && a->window == 0 && v.tree != nullptr && v.tree->words >= 1 && v.tree->pitch >= v.tree->words &&
           (static_cast<int64_t>(a->max_q) + 31) / 32 <= v.tree->words;
  return true;
}

// The call's geometry, as both the scratch size and the launch take it.
Plan prepare_attention(const pq_kv8_cache* c, const pq_kv8_attn* a, View& v, AttnArgs* p) {
  p->c = *c;
  p->a = without_idle_window(a);
  // Every token up to the query is in sight, or no sink is: plain attention, and its plan.  Half-precision outputs of a window that only
  // outlasts the texts keep the view's second half of a weight, so that they are as exact as once the texts have outgrown it (error 2.1e-4 of
  // the outputs' norm, without it 3.1e-4; us in a graph, with it and without, 32 / 8 heads of 128: 64 single tokens over 4000 106 / 103, 8 chunks
  // of 64 over 2000 82 / 75, 4 prompts of 2048 over 4096 509 / 403).
  const bool idle = v.kind == kSinks && (p->a.window == 0 || v.sinks == 0);
  const bool fine = v.kind != kPlain && !idle;
  if (idle && !(a->type == PQ_F16 && a->window > 0 && v.sinks > 0)) v.kind = kPlain;
  if (v.kind == kSinks && !idle) p->sinks = std::min(v.sinks, a->max_len);
  if (v.kind == kTree) {
    p->a.causal = 0;  // every token of the sequence, but for the bits
    p->tree = static_cast<const uint32_t*>(v.tree->bits_dev);
    p->tree_pitch = v.tree->pitch;
    p->tree_words = v.tree->words;
  }
  return plan_attention(c, &p->a, p, fine);
}

size_t scratch_bytes(const pq_kv8_cache* cache, const pq_kv8_attn* a, View v) {
  if (!valid_attn(cache, a) || !valid_view(a, v) || !countable(a) || a->B == 0 || a->max_q == 0) return 0;
  AttnArgs p = {};
  prepare_attention(cache, a, v, &p);
  return scratch_of(p);
}

pq_status attend(const pq_kv8_cache* cache, const void* q_dev, void* o_dev, const pq_kv8_attn* a, View v, void* scratch_dev,
                 size_t scratch_bytes, pq_stream_t stream) {
  if (!valid_attn(cache, a) || !valid_view(a, v)) return PQ_EINVAL;
  if (a->B == 0 || a->max_q == 0) return PQ_OK;
  const size_t e = bytes_of_type(a->type);
  if (q_dev == nullptr || o_dev == nullptr || a->cu_q_dev == nullptr || a->len_dev == nullptr ||
      (a->page_table_dev == nullptr && a->max_len > 0) || !is_aligned(q_dev, e) || !is_aligned(o_dev, e) ||
      !is_aligned(a->cu_q_dev, 4) || !is_aligned(a->len_dev, 4) || !is_aligned(a->page_table_dev, 4))
    return PQ_EINVAL;
  if (v.kind == kTree && (v.tree->bits_dev == nullptr || !is_aligned(v.tree->bits_dev, 4))) return PQ_EINVAL;
  if (!countable(a)) return PQ_EUNSUPPORTED;
  AttnArgs p = {};
  const Plan plan = prepare_attention(cache, a, v, &p);
  p.q = q_dev;
  p.o = o_dev;
  p.group = a->Hq / cache->Hkv;
  p.page_shift = cache->page_tokens == 16 ? 4 : cache->page_tokens == 32 ? 5 : cache->page_tokens == 64 ? 6 : 7;
  p.wide_q = is_aligned(q_dev, 16) && a->q_token_stride * e % 16 == 0 && a->q_head_stride * e % 16 == 0;
  p.wide_o = is_aligned(o_dev, 16) && a->o_token_stride * e % 16 == 0 && a->o_head_stride * e % 16 == 0;
  p.wait_limit_ns = wait_limit_ns();
  const size_t need = scratch_of(p);
  if (need > 0 && (scratch_dev == nullptr || scratch_bytes < need || !is_aligned(scratch_dev, 16))) return PQ_EINVAL;
  if (p.splits > 1 && !p.cluster) {
    const size_t parts = static_cast<size_t>(a->B) * a->max_q * a->Hq * p.splits;
    p.ml = static_cast<float2*>(scratch_dev);
    p.part = reinterpret_cast<float*>(p.ml + parts);
  }
  const int64_t units = static_cast<int64_t>(p.row_tiles) * p.splits * cache->Hkv;
  if (units > 0x7FFFFFFFll / a->B) return PQ_EUNSUPPORTED;
  const unsigned grid = static_cast<unsigned>(units * a->B);
  p.in_order = in_order(*a, plan, grid);
  p.err = device_error_word();
  if (p.err == nullptr) return PQ_ECUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t st;
  if (plan.tc)
    st = v.kind == kSinks  ? launch_attn_tc<kSinks>(p, grid, s)
         : v.kind == kTree ? launch_attn_tc<kTree>(p, grid, s)
                           : launch_attn_tc<kPlain>(p, grid, s);
  else
    st = v.kind == kSinks  ? launch_attn_rows<kSinks>(p, grid, plan.rows / 8, s)
         : v.kind == kTree ? launch_attn_rows<kTree>(p, grid, plan.rows / 8, s)
                           : launch_attn_rows<kPlain>(p, grid, plan.rows / 8, s);
  if (st == cudaSuccess && p.splits > 1 && !p.cluster) {
    if (a->type == PQ_F32)
      st = launch_join<float>(p, plan.rows, s);
    else if (a->type == PQ_F16)
      st = launch_join<__half>(p, plan.rows, s);
    else
      st = launch_join<__nv_bfloat16>(p, plan.rows, s);
  }
  return st == cudaSuccess && cudaGetLastError() == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

}  // namespace

// From about 40 query rows of a cache head on: a block's step costs the same for 1 to
// 128 rows here, and in pq_kv8_rows it grows with every 16 (D = 128, rows of a head, here
// against there: one sequence of 4000, 24 rows 21 / 21 us, 48 22 / 25; 32 sequences of 3000, 32 rows
// 111 / 87, 48 111 / 123, 64 112 / 150).
bool attn_tc_takes(const pq_kv8_cache& c, const pq_kv8_attn& a) {
  return a.type != PQ_F32 && c.D <= 128 && static_cast<int64_t>(a.max_q) * (a.Hq / c.Hkv) > 40;
}

}  // namespace pq

extern "C" {

size_t palquant_kv8_attention_scratch_bytes(const pq_kv8_cache* cache, const pq_kv8_attn* a) {
  return pq::scratch_bytes(cache, a, {pq::kPlain, 0, nullptr});
}

pq_status palquant_kv8_attention(const pq_kv8_cache* cache, const void* q_dev, void* o_dev, const pq_kv8_attn* a,
                                 void* scratch_dev, size_t scratch_bytes, pq_stream_t stream) {
  return pq::attend(cache, q_dev, o_dev, a, {pq::kPlain, 0, nullptr}, scratch_dev, scratch_bytes, stream);
}

size_t palquant_kv8_attention_sinks_scratch_bytes(const pq_kv8_cache* cache, const pq_kv8_attn* a, int32_t sinks) {
  return pq::scratch_bytes(cache, a, {pq::kSinks, sinks, nullptr});
}

pq_status palquant_kv8_attention_sinks(const pq_kv8_cache* cache, const void* q_dev, void* o_dev, const pq_kv8_attn* a,
                                       int32_t sinks, void* scratch_dev, size_t scratch_bytes, pq_stream_t stream) {
  return pq::attend(cache, q_dev, o_dev, a, {pq::kSinks, sinks, nullptr}, scratch_dev, scratch_bytes, stream);
}

size_t palquant_kv8_attention_tree_scratch_bytes(const pq_kv8_cache* cache, const pq_kv8_attn* a, const pq_kv8_tree* tree) {
  return pq::scratch_bytes(cache, a, {pq::kTree, 0, tree});
}

pq_status palquant_kv8_attention_tree(const pq_kv8_cache* cache, const void* q_dev, void* o_dev, const pq_kv8_attn* a,
                                      const pq_kv8_tree* tree, void* scratch_dev, size_t scratch_bytes, pq_stream_t stream) {
  return pq::attend(cache, q_dev, o_dev, a, {pq::kTree, 0, tree}, scratch_dev, scratch_bytes, stream);
}

}  // extern "C"
