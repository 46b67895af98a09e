// How the tensor-core kernel for 4-bit weights divides its memory and takes turns: host code too, so that it can be checked
// without a GPU.
//
// A job is 128 (groups of 128) or 64 of K.  Its weights and tokens come in a stage (128 of K), its unpacked weights take a slot, its
// groups' accumulators a place; each of these is used again after as many stages or jobs as there are.  A wait names the parity of
// the use it waits for, and an mbarrier answers it as well where the use before that one is still open.  So a warp that waits for a use
// must have waited for the one before: the warps that take jobs in turn divide the number of slots and places, and, as a set of
// unpacking warps takes every second stage, the number of stages is even.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define PQ_HOST_DEVICE __host__ __device__
#else
#define PQ_HOST_DEVICE
#endif

namespace pq {
namespace w4 {

constexpr int kBlockK = 128;                          // of K in a stage
constexpr int kWBytes = 8 * (1024 + 256);             // of a stage's weights at most: a tile's strips with four groups' fp32 scales
constexpr int kMaxStages = 8;
constexpr int kMaxSlots = 8;
constexpr uint32_t kAColumns = 256;                   // of tensor memory for unpacked weights; as many for accumulators
constexpr int kSmemBytes = 230400;                    // of 227 KB, beside the alignment and the static part

// GS: log2(group).  BN: tokens of a tile.  PARTS: of a token (three for fp32).
PQ_HOST_DEVICE constexpr int job_k(int GS) { return GS == 7 ? 128 : 64; }
PQ_HOST_DEVICE constexpr int jobs_of_stage(int GS) { return kBlockK / job_k(GS); }
PQ_HOST_DEVICE constexpr int slots(int GS) { return kAColumns / (job_k(GS) / 2); }
PQ_HOST_DEVICE constexpr int places(int BN, int GS) {
  return 256 / ((job_k(GS) >> GS) * BN) < kMaxSlots ? 256 / ((job_k(GS) >> GS) * BN) : kMaxSlots;
}
PQ_HOST_DEVICE constexpr int stage_bytes(int BN, int PARTS) { return kWBytes + BN * 256 * PARTS; }
// What the two sides of draining warps hand to one another at a tile's end.
PQ_HOST_DEVICE constexpr int exchange_bytes(int BN) { return BN < 128 ? BN * 512 : 0; }
PQ_HOST_DEVICE constexpr int stages(int BN, int PARTS) {
  return (kSmemBytes - exchange_bytes(BN)) / stage_bytes(BN, PARTS) < kMaxStages
             ? (kSmemBytes - exchange_bytes(BN)) / stage_bytes(BN, PARTS) / 2 * 2
             : kMaxStages;
}
PQ_HOST_DEVICE constexpr int smem_bytes(int BN, int PARTS) {
  return stages(BN, PARTS) * stage_bytes(BN, PARTS) + exchange_bytes(BN) + 1024 /* alignment */;
}

// Who takes jobs i, i + turns, i + 2 turns and so on: warps that issue MMAs, sets of warps that unpack, sides of warps that drain (with
// tiles of 128 tokens both sides drain every job).
PQ_HOST_DEVICE constexpr int issuers(int BN, int GS) { return places(BN, GS) < 4 ? places(BN, GS) : 4; }
PQ_HOST_DEVICE constexpr int unpacking_sets(int GS) { return 2 * jobs_of_stage(GS); }
PQ_HOST_DEVICE constexpr int draining_sides(int BN) { return BN == 128 ? 1 : 2; }

}  // namespace w4
}  // namespace pq
