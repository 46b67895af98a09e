"""Whether tensors of heads share memory: the rule that a call's checks use, compiled for the host, against every byte of many small
layouts, and at sizes past 64 bits (no GPU)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <random>
#include <set>
#include "pq_apart.h"
using namespace pq;

std::set<long> bytes_of(const HeadsAt& x, int tokens, int bytes) {
  std::set<long> all;
  for (int t = 0; t < tokens; ++t)
    for (int h = 0; h < x.heads; ++h)
      for (int i = 0; i < bytes; ++i) all.insert(static_cast<long>(x.at) + t * static_cast<long>(x.token_step) + h * static_cast<long>(x.head_step) + i);
  return all;
}

int main() {
  std::mt19937 rng(1);
  auto draw = [&](int lo, int hi) { return static_cast<int>(lo + rng() % (hi - lo + 1)); };
  long apart = 0, sharing = 0, beside = 0;
  for (int n = 0; n < 300000; ++n) {
    const int tokens = draw(1, 5), bytes = draw(1, 6);
    HeadsAt a{static_cast<uint64_t>(1000 + draw(-60, 60)), draw(0, 40), draw(0, 24), draw(1, 4)}, b{1000, draw(0, 40), draw(0, 24), draw(1, 4)};
    if (draw(0, 3)) b.token_step = a.token_step;
    if (draw(0, 2)) b.head_step = a.head_step;
    bool truth = false;
    const std::set<long> of_a = bytes_of(a, tokens, bytes);
    for (long byte : bytes_of(b, tokens, bytes)) truth = truth || of_a.count(byte);
    const bool says = heads_share(a, b, tokens, bytes);
    const bool exact = tokens == 1 || a.token_step == b.token_step;
    if (truth && !says || exact && truth != says || says != heads_share(b, a, tokens, bytes)) {
      std::printf("tokens %d bytes %d: a %ld %d %d %d, b %ld %d %d %d: %d, says %d\n", tokens, bytes, (long)a.at, (int)a.token_step, (int)a.head_step, (int)a.heads,
                  (long)b.at, (int)b.token_step, (int)b.head_step, (int)b.heads, truth, says);
      return 1;
    }
    const std::set<long> of_b = bytes_of(b, tokens, bytes);
    ++(says ? sharing : apart);
    beside += !says && *of_b.begin() < *of_a.rbegin() && *of_a.begin() < *of_b.rbegin();
  }
  if (apart < 1000 || sharing < 1000 || beside < 1000) return std::printf("%ld %ld %ld\n", apart, sharing, beside), 1;
  // steps near 2^63 elements of 4 bytes, and counts of 2^31
  const __int128 far = static_cast<__int128>(0x7FFFFFFFFFFFFFFFll) * 4;
  const HeadsAt x{1 << 20, far, far, 65535}, y{(1 << 20) + 256, far, far, 65535}, z{(1 << 20) + 255, far, far, 65535};
  if (heads_share(x, y, 0x7FFFFFFF, 256) || !heads_share(x, z, 0x7FFFFFFF, 256) || !same_heads(x, x, 5) || same_heads(x, y, 5)) return std::printf("far\n"), 1;
  // heads first, and a value's head between those of queries and keys
  const HeadsAt q{4096, 64, 64 << 20, 8}, k{4096 + (8ull << 26), 64, 64 << 20, 2}, packed_q{0, 3 * 64 * 8, 3 * 64, 8}, packed_k{64, 3 * 64 * 8, 3 * 64, 8};
  if (heads_share(q, k, 1 << 20, 64) || !heads_share(q, k, (1 << 20) + 1, 64) || heads_share(packed_q, packed_k, 1 << 20, 64) ||
      !heads_share(packed_q, packed_k, 2, 65))
    return std::printf("layouts\n"), 1;
  return 0;
}
"""


def test_shared_memory_of_heads(tmp_path):
    source, program = tmp_path / "apart.cc", tmp_path / "apart"
    source.write_text(PROGRAM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2208_01944_gb300", "csrc"), "-o", program, source])
    done = subprocess.run([program], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
