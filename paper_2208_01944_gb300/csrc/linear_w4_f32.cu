// The 4-bit dense layer for few tokens of this type.
#include "pq_w4_rows.cuh"

namespace pq {

template cudaError_t launch_w4_rows<float>(const W4Args& a, cudaStream_t stream);

}  // namespace pq
