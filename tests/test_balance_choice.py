"""The choice of a row's k largest logits in the balance loss: the order of csrc/choice_key.h, compiled for the host and walked as
the kernel walks it (softmax_ce_balance_kernel: the largest key below the choice before, k times)."""
import math
import os
import shutil
import struct
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1807_06629_b200", "csrc")
PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "choice_key.h"
using namespace prsgd;
int main(int argc, char** argv) {
  const int k = std::atoi(argv[1]), n = argc - 2;
  unsigned long long above = kChoiceAll;
  for (int j = 0; j < k; ++j) {
    unsigned long long best = 0;
    for (int c = 0; c < n; ++c) {
      const unsigned long long key = choice_key((uint32_t)std::strtoul(argv[2 + c], nullptr, 16), (uint32_t)c);
      if (key < above && key > best) best = key;
    }
    above = best;
    std::printf("%u ", best == 0 ? 0xFFFFFFFFu : choice_index(best));
  }
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    assert cxx
    d = tmp_path_factory.mktemp("choice")
    src, exe = d / "walk.cpp", d / "walk"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-I" + CSRC, str(src), "-o", str(exe)], check=True)

    def run(row, k):
        bits = [v if isinstance(v, str) else struct.pack(">f", v).hex() for v in row]
        return [int(c) for c in subprocess.run([str(exe), str(k), *bits], capture_output=True, text=True, check=True).stdout.split()]
    return run


def want(row, k):
    x = [math.nan if isinstance(v, str) else v for v in row]
    return sorted(range(len(x)), key=lambda c: (0, c) if math.isnan(x[c]) else (1, -x[c], c))[:k]


NAN, INF = math.nan, math.inf
ROWS = [[NAN, 1.0, 2.0, 0.5], [1.0, NAN, 2.0, NAN], [NAN] * 5, ["ffc00000", 3.0, "7f800001", "ffffffff"], [0.0, -0.0, 0.0, -0.0],
        [-INF] * 4, [INF, -INF, INF, 0.0, NAN], [3.4028234663852886e38, -3.4028234663852886e38, 1e-45, -1e-45, 0.0], [-1.0, -2.0, -1.0, -3.0], [7.0]]


@pytest.mark.parametrize("row", ROWS, ids=str)
def test_every_logit_can_be_chosen_once_nan_first(walk, row):
    for k in range(1, len(row) + 1):
        assert walk(row, k) == want(row, k)
