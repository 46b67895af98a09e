"""Reads in aligned words stay inside their row: the rule that the kernels use, compiled for the host, over all small rows."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "pq_words.h"
int main() {
  long reads = 0;
  for (int K = 1; K <= 300; ++K)
    for (int base = 0; base < 4; ++base)  // the row's address modulo 4
      for (int k = 0; k < K; k += 16) {
        const int off = (base + k) % 4;
        if (!pq::words_lie_in_row(k, K, off)) continue;
        ++reads;
        for (int byte = k - off; byte < k - off + 20; ++byte)
          if (byte < 0 || byte >= K) return std::printf("K %d base %d k %d reads byte %d\n", K, base, k, byte), 1;
        if (k - off > k || k - off + 20 < k + 16) return std::printf("K %d base %d k %d: bytes missing\n", K, base, k), 1;
      }
  std::printf("%ld\n", reads);
  return reads > 0 ? 0 : 1;
}
"""


def test_words_stay_in_the_row(tmp_path):
    source, program = tmp_path / "words.cc", tmp_path / "words"
    source.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2208_01944_gb300", "csrc"), "-o", program, source])
    done = subprocess.run([program], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout

