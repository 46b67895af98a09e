// Which bytes a read in aligned words touches: host code too, so that it can be checked without a GPU.
#pragma once

#ifdef __CUDACC__
#define PQ_HOST_DEVICE __host__ __device__
#else
#define PQ_HOST_DEVICE
#endif

namespace pq {

// Bytes [k, k + 16) of a row of K bytes as five aligned 32-bit words; `off` (0 to 3) is byte k's
// address modulo 4.  The words are bytes [k - off, k - off + 20): true if all of them are the row's own.
PQ_HOST_DEVICE constexpr bool words_lie_in_row(int k, int K, int off) { return k >= off && k - off + 20 <= K; }

}  // namespace pq
