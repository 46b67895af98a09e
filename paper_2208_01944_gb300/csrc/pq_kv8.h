// What the attention kernels over the 8-bit cache share on the host.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "palquant.h"

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
  int chunk;       // tokens of one part, a multiple of 16
  float2* ml;      // [B * max_q * Hq][splits]: running maximum and sum of every part
  float* part;     // [B * max_q * Hq][splits][D]: its unnormalised output
  unsigned int* err;
  bool wide_q, wide_o;  // rows on 16-byte boundaries
};

bool valid_kv8_cache(const pq_kv8_cache* c);

}  // namespace pq
