// The attention kernels over the 8-bit cache as they see a window, with the first tokens.
#include "pq_kv8_rows.cuh"
#include "pq_kv8_tiles.cuh"

namespace pq {

template cudaError_t launch_attn_rows<kSinks>(const AttnArgs& p, unsigned grid, int nt, cudaStream_t stream);
template cudaError_t launch_attn_tc<kSinks>(const AttnArgs& p, unsigned grid, cudaStream_t stream);

}  // namespace pq
