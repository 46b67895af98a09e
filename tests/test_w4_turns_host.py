"""Waits of the tensor-core kernel for 4-bit weights, role by role (no GPU).

An mbarrier wait names the parity of the use that it waits for, and is answered too while the use before it is still open.  So whoever
waits for a use of a stage, slot or place must have waited for the use before: here every warp that takes jobs in turn is walked
through its jobs, with the numbers that the kernel uses, compiled for the host."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <map>
#include "pq_w4_turns.h"
using namespace pq::w4;

int faults = 0;
// Whoever takes jobs first, first + step, ...; job i uses ring entry (i / per) % entries for the (i / per / entries)-th time.
void walk(const char* what, int first, int step, int per, int entries, int jobs, int BN, int GS, int PARTS) {
  std::map<int, int> last;  // of each entry, the use that was waited for last
  for (int i = first; i < jobs; i += step) {
    const int entry = i / per % entries, use = i / per / entries;
    const int before = last.count(entry) ? last[entry] : -1;
    if (use > before + 1) {
      std::printf("%s: tile of %d tokens, groups of 2^%d, %d parts: job %d waits for use %d of entry %d after use %d\n", what, BN, GS, PARTS, i, use, entry, before);
      ++faults;
      return;
    }
    last[entry] = use;
  }
}

void check(int BN, int GS, int PARTS) {
  const int per = jobs_of_stage(GS), jobs = 400 * per;
  for (int set = 0; set < unpacking_sets(GS); ++set) {
    walk("loaded", set, unpacking_sets(GS), per, stages(BN, PARTS), jobs, BN, GS, PARTS);
    walk("slot_empty", set, unpacking_sets(GS), 1, slots(GS), jobs, BN, GS, PARTS);
  }
  for (int w = 0; w < issuers(BN, GS); ++w) {
    walk("full", w, issuers(BN, GS), 1, slots(GS), jobs, BN, GS, PARTS);
    walk("acc_empty", w, issuers(BN, GS), 1, places(BN, GS), jobs, BN, GS, PARTS);
  }
  for (int side = 0; side < draining_sides(BN); ++side) walk("acc_full", side, draining_sides(BN), 1, places(BN, GS), jobs, BN, GS, PARTS);
  if (stages(BN, PARTS) < 2 || slots(GS) > kMaxSlots || places(BN, GS) > kMaxSlots || smem_bytes(BN, PARTS) + 1024 > 227 * 1024) {
    std::printf("tile of %d tokens, groups of 2^%d, %d parts: %d stages, %d slots, %d places, %d bytes\n", BN, GS, PARTS, stages(BN, PARTS), slots(GS), places(BN, GS), smem_bytes(BN, PARTS));
    ++faults;
  }
}

int main() {
  for (int GS = 5; GS <= 7; ++GS) {
    for (int BN : {32, 64, 128})
      if (BN < 128 || GS > 5) check(BN, GS, 1);
    check(32, GS, 3);
  }
  return faults;
}
"""


def test_every_wait_follows_the_wait_for_the_use_before(tmp_path):
    source, program = tmp_path / "turns.cc", tmp_path / "turns"
    source.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2208_01944_gb300", "csrc"), "-o", program, source])
    done = subprocess.run([program], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
