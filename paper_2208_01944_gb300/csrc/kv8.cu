// The paged 8-bit cache of keys and values: append (quantise in) and read (values
// out).  One scale covers a page's tokens of one head, so a block of threads owns
// a (page, head, side) at a time: it finds the scale of what the page will hold,
// rewrites the earlier codes where the scale grew, and writes the new ones.  New tokens
// stay in registers between the search for their largest magnitude and the rounding.
// Reading, a block takes several heads of a small page: the lookups (run, page) are three
// dependent loads (16 tokens a page, 8 x 2000 tokens of 8 heads of 128: 28 us one head
// a block, 18 us eight).
// Bound by HBM: each new element is read once and each code written once.  16 prompts of up to 4096
// tokens, 8 heads of 128, bf16: append 67 us, read 47 us (4.2 and 6.0 TB/s); the rest is the
// blocks' dependent lookups.
#include <cuda_runtime.h>

#include <algorithm>

#include "palquant.h"
#include "pq_internal.h"
#include "pq_tokens.cuh"

namespace pq {
namespace {

constexpr int kKvThreads = 256;

struct KvArgs {
  pq_kv8_cache c;
  pq_kv8_tokens t;
  const void* in[2];  // k, v (append)
  void* out[2];       // k, v (read); either may be NULL
  int blocks;         // pages of a sequence that a run can touch
  int heads;          // heads of one block of threads
  unsigned int* err;
  bool wide[2];  // rows of the float tensor on 16-byte boundaries
};

// What a block of threads works on: side, heads, and the run's tokens in one page.
struct KvUnit {
  int side, h, h_end;
  int64_t row;      // float row of the run's first token in the page
  int first, count; // slots [first, first + count) of the page belong to the run
  int64_t page;     // as the table has it
  bool there;       // false: nothing to do
};

__device__ __forceinline__ KvUnit kv_unit(const KvArgs& a) {
  KvUnit u;
  const int groups = (a.c.Hkv + a.heads - 1) / a.heads;
  const int b = blockIdx.y, blk = (blockIdx.x >> 1) / groups;
  u.side = blockIdx.x & 1;
  u.h = ((blockIdx.x >> 1) - blk * groups) * a.heads;
  u.h_end = min(u.h + a.heads, a.c.Hkv);
  const int T = a.c.page_tokens;
  const int start = a.t.start_dev[b], cu = a.t.cu_dev[b];
  const int n = min(a.t.cu_dev[b + 1] - cu, a.t.max_n);
  const int page = start / T + blk;
  const int64_t lo = max(static_cast<int64_t>(start), static_cast<int64_t>(page) * T);
  const int64_t hi = min(static_cast<int64_t>(start) + n, static_cast<int64_t>(page + 1) * T);
  u.there = false;
  if (start < 0 || n <= 0 || lo >= hi) return u;
  u.row = cu + (lo - start);
  u.first = static_cast<int>(lo - static_cast<int64_t>(page) * T);
  u.count = static_cast<int>(hi - lo);
  u.page = page < a.t.table_pitch ? a.t.page_table_dev[static_cast<int64_t>(b) * a.t.table_pitch + page] : -2;
  u.there = true;
  return u;
}

// False for a page that is not in the pool; reported.
__device__ __forceinline__ bool page_ok(const KvArgs& a, const KvUnit& u) {
  if (u.page >= 0 && u.page < a.c.num_pages) return true;
  if (threadIdx.x == 0) atomicOr(a.err, PQ_ERR_PAGE);
  return false;
}

// The vectors of a thread: v = threadIdx.x + i blockDim.x is piece `at` of row `row`, stepped
// along without a division a vector (only for loads that are all in flight together: in the read's
// loop the steps' chain cost 58 us instead of 53).
struct Walk {
  int D8, row, at, rows_on, pieces_on;
  __device__ explicit Walk(int d8)
      : D8(d8), row(threadIdx.x / d8), at(threadIdx.x % d8), rows_on(blockDim.x / d8), pieces_on(blockDim.x % d8) {}
  __device__ void next() {
    row += rows_on, at += pieces_on;
    if (at >= D8) at -= D8, ++row;
  }
};

// NV: vectors of 8 elements that a thread keeps; 0: the tokens are read twice.  Up to 64
// bytes of them, six blocks fit an SM (42 registers; with the 47 that the compiler would
// take five fit, and 16 prompts of up to 4096 tokens took 89 us instead of 71, now 67).
template <typename T, int NV>
__global__ void __launch_bounds__(kKvThreads, sizeof(T) * NV > 8 ? 1 : 6) pq_kv8_append(const __grid_constant__ KvArgs a) {
  __shared__ uint32_t red[8];
  const KvUnit u = kv_unit(a);
  if (!u.there) return;
  const int D8 = a.c.D / 8;
  const int64_t ts = u.side ? a.t.v_token_stride : a.t.k_token_stride;
  const int64_t hs = u.side ? a.t.v_head_stride : a.t.k_head_stride;
  const T* x = static_cast<const T*>(a.in[u.side]) + u.row * ts + u.h * hs;
  const bool wide = a.wide[u.side];
  const int nvec = u.count * D8;
  // the new tokens are on their way before the page's id is there
  Vec8<T> keep[NV > 0 ? NV : 1];
  if (NV > 0) {
    Walk w(D8);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (w.row < u.count) keep[i] = load8(x + w.row * ts + w.at * 8, 8, wide);
      w.next();
    }
  }
  if (!page_ok(a, u)) return;
  const int64_t slot0 = (u.page * a.c.Hkv + u.h) * a.c.page_tokens;
  int8_t* q = (u.side ? a.c.v_dev : a.c.k_dev) + slot0 * a.c.D;
  float* sp = (u.side ? a.c.v_scale_dev : a.c.k_scale_dev) + u.page * a.c.Hkv + u.h;
  const float was = u.first > 0 ? *sp : 0.0f;
  auto get = [&](int v) { return load8(x + (v / D8) * ts + (v % D8) * 8, 8, wide); };

  uint32_t top = 0;
  if (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (threadIdx.x + i * blockDim.x < nvec) top = max(top, amax8(keep[i]));
  } else {
    for (int v = threadIdx.x; v < nvec; v += blockDim.x) top = max(top, amax8(get(v)));
  }
  top = block_max(top, red);  // every thread has read the old scale before it
  const float fresh = scale_of_amax(top);
  const float scale = (fresh != fresh || was != was) ? __int_as_float(0x7FC00000) : fmaxf(was, fresh);
  const float inv = inverse_of_scale(scale);
  if (threadIdx.x == 0) *sp = scale;
  if (u.first > 0 && scale != was) {  // also where either is NaN
    const float ratio = __fmul_rn(was, inv);
    uint32_t* w = reinterpret_cast<uint32_t*>(q);
    for (int v = threadIdx.x; v < u.first * a.c.D / 4; v += blockDim.x) {
      float c[4];
      floats_of_codes(w[v], c);
      rounded_pair(c[0], c[1], ratio, c[0], c[1]);
      rounded_pair(c[2], c[3], ratio, c[2], c[3]);
      w[v] = ratio > 0.0f ? low_bytes(c[0], c[1], c[2], c[3]) : 0u;
    }
  }
  uint2* dst = reinterpret_cast<uint2*>(q + static_cast<int64_t>(u.first) * a.c.D);
  if (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = threadIdx.x + i * blockDim.x;
      if (v < nvec) dst[v] = codes8(keep[i], inv);
    }
  } else {
    for (int v = threadIdx.x; v < nvec; v += blockDim.x) dst[v] = codes8(get(v), inv);
  }
}

// 16-bit values: four loads of a thread before their stores, eight blocks an SM (16 prompts of up to
// 4096 tokens 53 -> 46 us, pages of 16 tokens 25 -> 18).  fp32 values: one (8 runs of 2000 tokens,
// 2 heads of 256: 17 us, four at a time 23).
template <typename T>
__global__ void __launch_bounds__(kKvThreads, sizeof(T) == 2 ? 8 : 1) pq_kv8_read(const __grid_constant__ KvArgs a) {
  constexpr int kLoads = sizeof(T) == 2 ? 4 : 1;
  const KvUnit u = kv_unit(a);
  if (!u.there || a.out[u.side] == nullptr || !page_ok(a, u)) return;
  const int D8 = a.c.D / 8;
  const int64_t ts = u.side ? a.t.v_token_stride : a.t.k_token_stride;
  const int64_t hs = u.side ? a.t.v_head_stride : a.t.k_head_stride;
  T* rows = static_cast<T*>(a.out[u.side]) + u.row * ts;
  const int8_t* codes = u.side ? a.c.v_dev : a.c.k_dev;
  const float* scales = (u.side ? a.c.v_scale_dev : a.c.k_scale_dev) + u.page * a.c.Hkv;
  const bool wide = a.wide[u.side];
  for (int h = u.h; h < u.h_end; ++h) {
    const int64_t slot0 = (u.page * a.c.Hkv + h) * a.c.page_tokens + u.first;
    const uint2* q = reinterpret_cast<const uint2*>(codes + slot0 * a.c.D);
    const float scale = scales[h];
    T* x = rows + h * hs;
    const int nvec = u.count * D8, step = blockDim.x;
    for (int v0 = threadIdx.x; v0 < nvec; v0 += kLoads * step) {
      uint2 c[kLoads];
#pragma unroll
      for (int k = 0; k < kLoads; ++k)
        if (v0 + k * step < nvec) c[k] = q[v0 + k * step];
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        const int v = v0 + k * step;
        if (v >= nvec) break;
        float f[2][4];
        floats_of_codes(c[k].x, f[0]);
        floats_of_codes(c[k].y, f[1]);
        Vec8<T> r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = from_f32<T>(__fmul_rn(f[i >> 2][i & 3], scale));
        store8(x + (v / D8) * ts + (v % D8) * 8, r, 8, wide);
      }
    }
  }
}

// Threads of a block: about four of the vectors of 8 that a page and head can receive
// for each, so that small pages leave an SM as many bytes in flight as large ones.
int threads_of(const KvArgs& a) {
  const int tokens = a.c.page_tokens < a.t.max_n ? a.c.page_tokens : a.t.max_n;
  const int vecs = tokens * (a.c.D / 8);
  return vecs <= 256 ? 64 : vecs <= 512 ? 128 : kKvThreads;
}

template <typename T>
void launch_append(const KvArgs& a, dim3 grid, cudaStream_t s) {
  const int threads = threads_of(a);
  const int tokens = a.c.page_tokens < a.t.max_n ? a.c.page_tokens : a.t.max_n;
  const int nv = (tokens * (a.c.D / 8) + threads - 1) / threads;
  if (nv <= 1)
    pq_kv8_append<T, 1><<<grid, threads, 0, s>>>(a);
  else if (nv <= 2)
    pq_kv8_append<T, 2><<<grid, threads, 0, s>>>(a);
  else if (nv <= 4)
    pq_kv8_append<T, 4><<<grid, threads, 0, s>>>(a);
  else if (nv <= 8)
    pq_kv8_append<T, 8><<<grid, threads, 0, s>>>(a);
  else
    pq_kv8_append<T, 0><<<grid, threads, 0, s>>>(a);
}

}  // namespace

bool valid_kv8_cache(const pq_kv8_cache* c) {
  return c != nullptr && c->num_pages >= 1 && c->Hkv >= 1 &&
         (c->page_tokens == 16 || c->page_tokens == 32 || c->page_tokens == 64 || c->page_tokens == 128) &&
         c->D >= 16 && c->D <= 256 && c->D % 16 == 0 && c->k_dev != nullptr && c->v_dev != nullptr &&
         c->k_scale_dev != nullptr && c->v_scale_dev != nullptr && is_aligned(c->k_dev, 16) &&
         is_aligned(c->v_dev, 16) && is_aligned(c->k_scale_dev, 4) && is_aligned(c->v_scale_dev, 4);
}

namespace {

// Checks what both calls share and fills the launch; an empty grid: nothing to do.
pq_status kv_args(const pq_kv8_cache* c, const pq_kv8_tokens* t, const void* k, const void* v, bool reading, KvArgs* a,
                  dim3* grid) {
  *grid = dim3(0);
  if (!valid_kv8_cache(c) || t == nullptr) return PQ_EINVAL;
  if (t->type != PQ_F32 && t->type != PQ_F16 && t->type != PQ_BF16) return PQ_EINVAL;
  if (t->B < 0 || t->max_n < 0 || t->table_pitch < 0) return PQ_EINVAL;
  if (t->B == 0 || t->max_n == 0) return PQ_OK;
  if (t->cu_dev == nullptr || t->start_dev == nullptr || t->page_table_dev == nullptr || !is_aligned(t->cu_dev, 4) ||
      !is_aligned(t->start_dev, 4) || !is_aligned(t->page_table_dev, 4))
    return PQ_EINVAL;
  const size_t e = bytes_of_type(t->type);
  if (!is_aligned(k, e) || !is_aligned(v, e)) return PQ_EINVAL;
  if (t->k_token_stride < 0 || t->k_head_stride < 0 || t->v_token_stride < 0 || t->v_head_stride < 0) return PQ_EINVAL;
  a->c = *c;
  a->t = *t;
  a->wide[0] = is_aligned(k, 16) && t->k_token_stride * e % 16 == 0 && t->k_head_stride * e % 16 == 0;
  a->wide[1] = is_aligned(v, 16) && t->v_token_stride * e % 16 == 0 && t->v_head_stride * e % 16 == 0;
  a->blocks = static_cast<int>((static_cast<int64_t>(t->max_n) + c->page_tokens - 2) / c->page_tokens + 1);
  a->err = device_error_word();
  if (a->err == nullptr) return PQ_ECUDA;
  // heads that a block reads: up to 2048 vectors of 8, as long as that leaves eight blocks
  // for every SM of the chip
  const int vecs = std::min(c->page_tokens, t->max_n) * (c->D / 8);
  const int64_t pages = 2ll * a->blocks * t->B;
  a->heads = reading ? std::min(c->Hkv, std::max(1, 2048 / vecs)) : 1;
  while (a->heads > 1 && pages * ((c->Hkv + a->heads - 1) / a->heads) < 8 * 152) a->heads = (a->heads + 1) / 2;
  const int64_t units = 2ll * ((c->Hkv + a->heads - 1) / a->heads) * a->blocks;
  if (units > 0x7FFFFFFFll || t->B > 65535) return PQ_EUNSUPPORTED;
  *grid = dim3(static_cast<unsigned>(units), static_cast<unsigned>(t->B));
  return PQ_OK;
}

}  // namespace
}  // namespace pq

extern "C" {

pq_status palquant_kv8_append(const pq_kv8_cache* cache, const void* k_dev, const void* v_dev,
                              const pq_kv8_tokens* t, pq_stream_t stream) {
  if (t != nullptr && t->B > 0 && t->max_n > 0 && (k_dev == nullptr || v_dev == nullptr)) return PQ_EINVAL;
  pq::KvArgs a = {};
  dim3 grid(0);
  const pq_status st = pq::kv_args(cache, t, k_dev, v_dev, false, &a, &grid);
  if (st != PQ_OK || grid.x == 0) return st;
  a.in[0] = k_dev;
  a.in[1] = v_dev;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (t->type == PQ_F32)
    pq::launch_append<float>(a, grid, s);
  else if (t->type == PQ_F16)
    pq::launch_append<__half>(a, grid, s);
  else
    pq::launch_append<__nv_bfloat16>(a, grid, s);
  return cudaGetLastError() == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

pq_status palquant_kv8_read(const pq_kv8_cache* cache, void* k_dev, void* v_dev, const pq_kv8_tokens* t,
                            pq_stream_t stream) {
  if (t != nullptr && t->B > 0 && t->max_n > 0 && k_dev == nullptr && v_dev == nullptr) return PQ_EINVAL;
  pq::KvArgs a = {};
  dim3 grid(0);
  const pq_status st = pq::kv_args(cache, t, k_dev, v_dev, true, &a, &grid);
  if (st != PQ_OK || grid.x == 0) return st;
  a.out[0] = k_dev;
  a.out[1] = v_dev;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (t->type == PQ_F32)
    pq::pq_kv8_read<float><<<grid, pq::threads_of(a), 0, s>>>(a);
  else if (t->type == PQ_F16)
    pq::pq_kv8_read<__half><<<grid, pq::threads_of(a), 0, s>>>(a);
  else
    pq::pq_kv8_read<__nv_bfloat16><<<grid, pq::threads_of(a), 0, s>>>(a);
  return cudaGetLastError() == cudaSuccess ? PQ_OK : PQ_ECUDA;
}

}  // extern "C"
