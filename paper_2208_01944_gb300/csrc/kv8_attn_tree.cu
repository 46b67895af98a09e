// The attention kernels over the 8-bit cache as they see the text, and the drafts that the query's bits name.
#include "pq_kv8_rows.cuh"
#include "pq_kv8_tiles.cuh"

namespace pq {

template cudaError_t launch_attn_rows<kTree>(const AttnArgs& p, unsigned grid, int nt, cudaStream_t stream);
template cudaError_t launch_attn_tc<kTree>(const AttnArgs& p, unsigned grid, cudaStream_t stream);

}  // namespace pq
