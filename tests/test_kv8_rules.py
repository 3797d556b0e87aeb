"""Rules by sizes of the 8-bit cache's host side (host code, no GPU)."""
from __future__ import annotations

import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_11517_amd", "csrc")
PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "k8_rules.hpp"
int main(int argc, char** argv) {
  for (int i = 1; i + 1 < argc; i += 2) std::printf("%d ", k8::append_group(std::atoll(argv[i]), std::atoi(argv[i + 1])));
}
"""


@pytest.fixture(scope="module")
def append_group(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", f"-I{CSRC}", str(d / "rules.cpp"), "-o", str(d / "rules")], check=True)

    def ask(*sizes):
        r = subprocess.run([str(d / "rules"), *(str(x) for s in sizes for x in s)], capture_output=True, text=True, check=True)
        return [int(x) for x in r.stdout.split()]
    return ask


def test_rows_to_a_work_group_of_append(append_group):
    """By rows and heads alone: one row for small steps, a whole block's for prompts."""
    assert append_group((1, 8), (333, 8), (334, 8), (666, 8), (667, 8), (1600, 8), (1601, 8), (4096, 8), (4097, 8), (8192, 8)) == [1, 1, 2, 2, 4, 4, 8, 8, 16, 16]
    assert append_group((1333, 1), (1334, 1), (1 << 28, 1), (0, 1), (1, 256), (21, 256)) == [1, 2, 16, 1, 1, 4]


def test_the_cases_of_the_gpu_tests_reach_every_size(append_group):
    from test_gpu_kv8_append_groups import SIZES

    assert append_group(*((n, h) for n, h, _ in SIZES)) == [g for _, _, g in SIZES]
    assert {g for _, _, g in SIZES} == {1, 2, 4, 8, 16}


SPLIT = r"""
#include <cstdio>
#include "k8_split.hpp"
// every tile up to 100 chunks, a part of them plain, for pieces of 256 tokens (cost 4) and longer
int main() {
  int shortest = 1 << 20;
  for (int chunks = 1; chunks <= 100; ++chunks)
    for (int cheap = 0; cheap <= chunks; ++cheap)
      for (int most = 2 * k8::kLeastAlone / k8::kChunkTokens; most <= 64; ++most) {
        const k8::Cost c{chunks, cheap};
        const int parts = k8::pieces_of(c.all(), most);
        if (c.all() > parts * most || (parts > 1 && 2 * c.all() <= parts * most)) return 1;  // at most `most` on the mean, more than half of it
        int at = 0;
        if (parts > 1)
          for (int k = 0; k < parts; ++k) {
            const int lo = k8::piece_at(c, k, parts), hi = k + 1 < parts ? k8::piece_at(c, k + 1, parts) : chunks;
            if (lo != at || hi <= lo) return 2;  // one behind the other, none empty
            const int cost = 2 * (hi < cheap ? hi : cheap) - 2 * (lo < cheap ? lo : cheap) + 3 * (hi > cheap ? hi - cheap : 0) - 3 * (lo > cheap ? lo - cheap : 0);
            if (cost > most + 2) return 3;  // a chunk more at most, less what it was begun with
            if (hi - lo < shortest) shortest = hi - lo;
            at = hi;
          }
        if (parts > 1 && at != chunks) return 4;
      }
  const k8::Cost c{7, 7};  // 769 tokens: the last chunk holds one
  for (int k = 0; k < 4; ++k) std::printf("%d ", k8::piece_at(c, k, k8::pieces_of(c.all(), 4)));
  std::printf("%d\n", shortest);
}
"""


def test_pieces_of_a_tiles_tokens(tmp_path):
    """What the split guarantees: every chunk in one piece, none without, on the mean more than half of the length that is aimed at -- and no more than that."""
    (tmp_path / "split.cpp").write_text(SPLIT)
    subprocess.run(["g++", "-std=c++17", "-D__device__=", f"-I{CSRC}", str(tmp_path / "split.cpp"), "-o", str(tmp_path / "split")], check=True)
    r = subprocess.run([str(tmp_path / "split")], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.split() == ["0", "1", "3", "5", "1"], (r.returncode, r.stdout)
