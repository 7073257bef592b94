"""Which variants the group norm's rule chooses, without a GPU: the GPU tests' shapes reach every way that a call can
take, so a changed rule fails here and not by leaving one untested."""
import ctypes as C
import os
import subprocess

import pytest

from test_gpu_norm import SHAPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1805_11144_amd", "csrc")

SHIM = r'''
#include "operators_rules.hpp"
using namespace ms;
extern "C" void norm_rule(int64_t batch, int64_t positions, int64_t groups, int64_t nw, int64_t grad, int64_t* out) {
  const NormShape s = norm_shape(batch, positions, groups, nw, grad != 0);
  out[0] = s.team, out[1] = s.words, out[2] = s.lanes, out[3] = s.runs, out[4] = s.run, out[5] = s.wide;
}
'''


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Wextra", "-Werror", "-I", CSRC,
                    str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    lib = C.CDLL(str(d / "shim.so"))

    def call(batch, positions, groups, nw, grad):
        out = (C.c_int64 * 6)()
        lib.norm_rule(*[C.c_int64(x) for x in (batch, positions, groups, nw, grad)], out)
        return dict(zip(("team", "words", "lanes", "runs", "run", "wide"), out))
    return call


def words_of(width, elem):
    v = 16 // elem
    while width % v:
        v //= 2
    return width // v


def test_every_way_is_reached(rule):
    """(a team of several wavefronts, or 0: runs, -1; words of a thread; one position)"""
    seen = {0: set(), 1: set()}
    for elem in (2, 4):
        for b, t, g, w in SHAPES:
            for grad in (0, 1):
                s = rule(b, t, g, words_of(w, elem), grad)
                seen[grad].add((s["team"] > 64, s["words"], t == 1) if s["team"] else "runs")
    teams = {(False, 1), (False, 2), (False, 4), (True, 2), (True, 4)}
    assert {x[:2] for x in seen[0] if x != "runs"} == teams and {x[:2] for x in seen[1] if x != "runs"} == teams
    assert {x[2] for x in seen[0] if x != "runs"} == {True, False} and {x[2] for x in seen[1] if x != "runs"} == {True}
    assert "runs" in seen[0] and "runs" in seen[1]


@pytest.mark.parametrize("b,t,g,nw", [(0, 0, 1, 1), (1, 0, 3, 5), (0, 7, 3, 5), (1, 1, 1, 1), (13, 777, 9, 37), (1, (1 << 31) - 1, 1, 1),
                                      ((1 << 31) - 1, 1, 1, 1), (16384, 5, 2, 700), (1, 1, (1 << 24) - 1, 1), (3, 1, 1, 1 << 23)])
def test_runs_cover_all_positions(rule, b, t, g, nw):
    for grad in (0, 1):
        s = rule(b, t, g, nw, grad)
        if s["team"]:
            assert s["team"] in (1, 2, 4, 8, 16, 32, 64, 256) and s["team"] * s["words"] >= t * nw and s["words"] in (1, 2, 4)
            assert 1 <= s["lanes"] <= max(b, 1)
        else:
            assert s["run"] >= 1 and s["run"] * s["runs"] >= t and (s["runs"] == 0 or s["run"] * (s["runs"] - 1) < t)
            assert 1 <= s["wide"] <= 256
