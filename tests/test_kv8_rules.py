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
