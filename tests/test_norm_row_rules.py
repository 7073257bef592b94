"""The group norm's rule on many batch rows, without a GPU: the GPU tests' shapes reach teams that go through several rows
and write out several sums, and joins of two and three steps; no team adds up more than 64 rows one after the other."""
import ctypes as C
import subprocess

import pytest

from test_gpu_norm_rows import RUNS, TEAMS
from test_norm_rules import CSRC, SHIM, words_of

COLUMN_ROWS = 512   # of a step of the join


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "shim.cpp").write_text(SHIM.replace("norm_rule", "norm_rule7").replace("out[0] = ", "out[6] = s.pieces, out[0] = "))
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Wextra", "-Werror", "-I", CSRC,
                    str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    lib = C.CDLL(str(d / "shim.so"))

    def call(batch, positions, groups, nw, grad):
        out = (C.c_int64 * 7)()
        lib.norm_rule7(*[C.c_int64(x) for x in (batch, positions, groups, nw, grad)], out)
        return dict(zip(("team", "words", "lanes", "runs", "run", "wide", "pieces"), out))
    return call


def steps(rows):
    n = 1
    while rows > COLUMN_ROWS:
        rows, n = -(-rows // COLUMN_ROWS), n + 1
    return n


def test_shapes_reach_the_ways(rule):
    seen = set()
    for elem in (2, 4):
        for b, t, g, w in TEAMS + RUNS:
            s = rule(b, t, g, words_of(w, elem), 1)
            assert bool(s["team"]) == (t == 1 and words_of(w, elem) <= 1024)
            if s["team"]:
                at_once = 4 if s["words"] * words_size(w, elem) <= 16 else 2 if s["words"] * words_size(w, elem) <= 32 else 1
                rows = -(-b // s["lanes"])
                seen.add(("wide" if s["team"] > 64 else "team", "rounds" if rows > at_once else "one"))
                seen.add(("team steps", steps(s["lanes"] * s["pieces"])))
                seen.add(("pieces", min(s["pieces"], 2)))
                if rows > at_once and b % (at_once * s["lanes"]):
                    seen.add("a last round that is not full")
            else:
                seen.add(("run steps", steps(b * s["runs"])))
    assert seen >= {("team", "rounds"), ("wide", "rounds"), ("team", "one"), ("team steps", 1), ("team steps", 2),
                    ("run steps", 2), ("run steps", 3), "a last round that is not full", ("pieces", 1), ("pieces", 2)}


def words_size(width, elem):
    return elem * width // words_of(width, elem)


@pytest.mark.parametrize("b,g,nw", [(16384, 16, 16), (1 << 20, 16, 16), (1 << 24, 1, 1), (100, 4096, 2), (1 << 20, 4096, 2),
                                    (1 << 17, 1 << 14, 1), ((1 << 31) - 1, 1, 1)])
def test_rows_of_a_team_and_the_grid(rule, b, g, nw):
    s = rule(b, 1, g, nw, 1)
    assert s["lanes"] * g * s["team"] <= 1 << 31
    assert s["lanes"] * s["pieces"] * 64 >= b and (s["pieces"] == 1 or s["lanes"] * (s["pieces"] - 1) * 64 < b)
