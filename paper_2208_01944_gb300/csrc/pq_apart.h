// Whether two tensors of heads share memory: host code alone, so that it can be checked without a GPU.
#pragma once

#include <cstdint>

namespace pq {

// Heads of `bytes` bytes each: that of token t and head h begins at at + t * token_step + h * head_step (bytes, 0 and up).
struct HeadsAt {
  uint64_t at;
  __int128 token_step, head_step;
  int64_t heads;
};

// The same heads in the same places (the step of a dimension of one does not count).
inline bool same_heads(const HeadsAt& a, const HeadsAt& b, int64_t tokens) {
  return a.at == b.at && a.heads == b.heads && (tokens <= 1 || a.token_step == b.token_step) && (a.heads <= 1 || a.head_step == b.head_step);
}

// Whether some head of `a` shares a byte with some head of `b`, `tokens` tokens each.  Exact for tensors that lie apart as a whole and for those
// of one token step, in time that grows with the heads; others that reach into one another's memory count as sharing.
inline bool heads_share(const HeadsAt& a, const HeadsAt& b, int64_t tokens, int64_t bytes) {
  if (a.heads <= 0 || b.heads <= 0 || tokens <= 0) return false;
  const __int128 last = tokens - 1, off = static_cast<__int128>(b.at) - static_cast<__int128>(a.at);  // of b's first byte from a's
  const __int128 row_a = (a.heads - 1) * a.head_step + bytes, row_b = (b.heads - 1) * b.head_step + bytes;  // a token's heads, ends included
  if (off >= last * a.token_step + row_a || -off >= last * b.token_step + row_b) return false;
  if (tokens > 1 && a.token_step != b.token_step) return true;
  const __int128 step = tokens > 1 ? a.token_step : 0;
  if (step > 0) {
    const __int128 column = (off % step + step) % step;  // where b's rows begin in a's
    if (column >= row_a && column + row_b <= step) return false;
  }
  // a head of b at `at` bytes from one of a, of the same token: whether they meet, or do so some tokens on
  auto meet = [&](__int128 at) {
    if (step == 0) return at < bytes && -at < bytes;
    const __int128 from = at < 0 ? -at / step : -((at + step - 1) / step);  // at + from * step is the first that is not above 0 ...
    for (__int128 t = from; t <= from + 1; ++t) {                          // ... and the next one the last that is not below
      const __int128 moved = at + (t < -last ? -last : t > last ? last : t) * step;
      if (moved < bytes && -moved < bytes) return true;
    }
    return false;
  };
  if (a.heads == 1 || b.heads == 1 || a.head_step == b.head_step) {
    const __int128 head_step = b.heads == 1 ? a.head_step : b.head_step;
    for (int64_t i = 1 - a.heads; i < b.heads; ++i)
      if (meet(off + i * head_step)) return true;
    return false;
  }
  if (a.heads > 65536 / b.heads) return true;
  for (int64_t i = 0; i < a.heads; ++i)
    for (int64_t j = 0; j < b.heads; ++j)
      if (meet(off + j * b.head_step - i * a.head_step)) return true;
  return false;
}

}  // namespace pq
