"""How calls of the vocabulary loss are cut up (csrc/vocab_plan.h, compiled for the host): what must hold for every call, and that the sizes of
vocab_shapes.py reach the branches that they are there for."""
import os
import random
import shutil
import subprocess

import pytest

import vocab_shapes as shapes

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1807_06629_b200", "csrc")
FIELDS = ["Tp", "tm", "tiles", "td", "kd", "tasks", "longest", "run", "runs", "piece", "pieces", "gp", "seqs", "parts", "kpart", "run_w", "h_first",
          "last_tiles", "last_blocks", "lag", "slots"]
FORMS = ["few", "few_grad"]
PROGRAM = r"""
#include <cstdio>
#include "vocab_plan.h"
int main() {
  int split, grad, D;
  long long G, T, V;
  while (std::scanf("%d %d %lld %lld %lld %d", &split, &grad, &G, &T, &V, &D) == 6) {
    const prsgd::VocabCuts c = prsgd::vocab_cuts(split, grad, G, T, V, D);
    std::printf(""" + '"' + "%lld " * len(FIELDS + FORMS) + r"\n" + '"' + "".join(", (long long)c." + f for f in FIELDS) + r""", (long long)prsgd::vocab_few(split, G, T, V, D), (long long)prsgd::vocab_few_grad(T, D));
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "plan.cpp", d / "plan"
    src.write_text(PROGRAM)
    subprocess.run([shutil.which("g++") or "c++", "-std=c++17", "-I" + CSRC, str(src), "-o", str(exe)], check=True)

    def run(calls):
        text = "\n".join(" ".join(str(int(x)) for x in c) for c in calls)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        return [dict(zip(FIELDS + FORMS, map(int, line.split()))) for line in out]
    return run


def up(a, b):
    return -(-a // b)


def test_every_call_is_covered_once(plans):
    """Tiles, pieces, parts and runs cover the vocabulary and the contractions, without an empty piece, and what a call waits for lies in earlier phases."""
    rng = random.Random(5)
    log = lambda hi: int(round(2 ** rng.uniform(0, hi)))          # noqa: E731
    calls = [(rng.random() < 0.5, rng.random() < 0.7, log(12), log(22), log(24), log(16)) for _ in range(4000)]
    calls += [(s, 1, 1, T, V, D) for s in (0, 1) for T in (1, 64, 65, 1 << 22) for V in (1, 255, 257, 1 << 24) for D in (1, 64, 65536)]
    for (split, grad, G, T, V, D), c in zip(calls, plans(calls)):
        if G * T * V > 1 << 44:
            continue                                       # (more tiles than a call takes: refused)
        assert c["Tp"] >= T and c["Tp"] % 64 == 0 and c["tiles"] == up(V, 256) and c["td"] == up(D, 256) and c["kd"] == up(D, 64)
        if not grad:
            assert 1 <= c["run"] <= 8 and (c["runs"] - 1) * c["run"] < c["tiles"] <= c["runs"] * c["run"]
            continue
        piece, n = c["piece"], c["pieces"]
        assert piece % 256 == 0 and (n - 1) * piece < V <= n * piece and c["seqs"] == G * n
        assert c["gp"] % 64 == 0 and min(piece, V) <= c["gp"] <= piece
        assert c["last_tiles"] == up(V - (n - 1) * piece, 256) and c["last_blocks"] == up(V - (n - 1) * piece, 64)
        assert 1 <= c["parts"] <= 32 and c["parts"] * c["kpart"] * 64 >= min(piece, V) and c["kpart"] <= 256
        assert 1 <= c["run_w"] <= 8 and 1 <= c["lag"] <= c["seqs"] and c["slots"] == min(c["seqs"], 2 * c["lag"] + 1)
        assert c["longest"] == (not split and max(T, D) > 8192)


def test_sizes_reach_their_branches(plans):
    both = [0, 1]
    for shape in shapes.RUNS_OF_DW:
        for c in plans([(s, 1, *shape) for s in both]):
            assert c["run_w"] > 1 and c["tiles"] % c["run_w"] != 0 and c["pieces"] == 1 and c["parts"] > 1 and not c["longest"], (shape, c)
    assert {c["td"] > 1 for c in plans([(0, 1, *s) for s in shapes.RUNS_OF_DW])} == {False, True}
    for shape in shapes.PIECES:
        for c in plans([(s, 1, *shape) for s in both]):
            assert c["pieces"] > 1 and c["parts"] > 1 and c["td"] > 1 and c["tm"] > 1 and c["last_tiles"] < c["piece"] // 256 and not c["longest"], (shape, c)
    wide, deep = plans([(0, 1, *s) for s in shapes.LONG])
    assert wide["longest"] and wide["pieces"] > 1 and wide["parts"] > 1 and wide["td"] > 1 and wide["tm"] > 32
    assert deep["longest"] and deep["kd"] > 128 and deep["parts"] > 1
    for shape in shapes.RUNS_OF_LOSS:
        for c in plans([(s, 0, *shape) for s in both]):
            assert c["run"] > 1 and c["tiles"] % c["run"] != 0 and c["kd"] > 8, (shape, c)


def test_forms_of_few_tokens(plans):
    for shapes_, want in ((shapes.FEW, 1), (shapes.NOT_FEW, 0)):
        assert [c["few"] for c in plans([(0, 0, *s) for s in shapes_])] == [want] * len(shapes_)
        assert all(c["few"] for c in plans([(1, 0, *s) for s in shapes_]))
    # fp32: up to eight tokens, up to the columns that the contract names
    for T, D, want in ((2, 12288, 1), (2, 12289, 0), (1, 24576, 1), (1, 24577, 0), (3, 6144, 1), (8, 6144, 1), (8, 6145, 0), (9, 64, 0)):
        assert plans([(1, 0, 1, T, 1000, D)])[0]["few"] == want, (T, D)
    for T, D, want in ((1, 2048, 1), (2, 2048, 1), (2, 2049, 0), (3, 8, 0)):
        assert plans([(s, 1, 1, T, 1000, D) for s in (0, 1)])[0]["few_grad"] == want, (T, D)
