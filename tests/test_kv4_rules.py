"""Rules of the 4-bit cache's host side and plan, compiled for the CPU."""
from __future__ import annotations

import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_11517_amd", "csrc")

SPLIT = r"""
#include <algorithm>
#include <cstdio>
#include "k8_split.hpp"
// every tile up to 200 chunks, a part of them plain, for pieces of 128 tokens (cost 2) and longer
int main() {
  for (int chunks = 1; chunks <= 200; ++chunks)
    for (int cheap = 0; cheap <= chunks; ++cheap)
      for (int most = 2 * k8::kLeastAlone4 / k8::kChunkTokens; most <= 64; ++most) {
        const k8::Cost c{chunks, cheap};
        int parts = k8::pieces_of(c.all(), most);
        if (most < 2 * k8::kLeastAlone / k8::kChunkTokens) parts = std::min(parts, k8::most_pieces(c));
        if (parts < 1 || parts > chunks) return 1;  // what the launch has room for
        int at = 0;
        for (int k = 0; k < parts && parts > 1; ++k) {
          const int lo = k8::piece_at(c, k, parts), hi = k + 1 < parts ? k8::piece_at(c, k + 1, parts) : chunks;
          if (lo != at || hi <= lo) return 2;  // one behind the other, none empty
          at = hi;
        }
        if (parts > 1 && at != chunks) return 3;
        if (most < 4 && cheap == chunks && parts != (2 * chunks + most - 1) / most) return 4;  // plain tokens go in as many as are aimed at
      }
  return 0;
}
"""


def test_pieces_of_a_tiles_tokens(tmp_path):
    (tmp_path / "split.cpp").write_text(SPLIT)
    subprocess.run(["g++", "-std=c++17", "-D__device__=", f"-I{CSRC}", str(tmp_path / "split.cpp"), "-o", str(tmp_path / "split")], check=True)
    assert subprocess.run([str(tmp_path / "split")]).returncode == 0
