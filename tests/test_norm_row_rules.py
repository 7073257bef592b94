"""The group norm's rule on many batch rows, without a GPU: the GPU tests' shapes reach teams that go through several rows
and joins of two and three steps, and no thread adds up more than 64 rows one after the other."""
import pytest

from test_gpu_norm_rows import RUNS, TEAMS
from test_norm_rules import rule, words_of  # noqa: F401  (rule: a fixture)

COLUMN_ROWS = 512   # of a step of the join


def steps(rows):
    n = 1
    while rows > COLUMN_ROWS:
        rows, n = -(-rows // COLUMN_ROWS), n + 1
    return n


def test_shapes_reach_the_ways(rule):  # noqa: F811
    seen = set()
    for elem in (2, 4):
        for b, t, g, w in TEAMS + RUNS:
            s = rule(b, t, g, words_of(w, elem), 1)
            assert bool(s["team"]) == (t == 1 and words_of(w, elem) <= 1024)
            if s["team"]:
                at_once = 4 if s["words"] * words_size(w, elem) <= 16 else 2 if s["words"] * words_size(w, elem) <= 32 else 1
                rows = -(-b // s["lanes"])
                seen.add(("wide" if s["team"] > 64 else "team", "rounds" if rows > at_once else "one"))
                seen.add(("team steps", steps(s["lanes"])))
                if rows > at_once and b % (at_once * s["lanes"]):
                    seen.add("a last round that is not full")
            else:
                seen.add(("run steps", steps(b * s["runs"])))
    assert seen >= {("team", "rounds"), ("wide", "rounds"), ("team", "one"), ("team steps", 1), ("team steps", 2),
                    ("run steps", 2), ("run steps", 3), "a last round that is not full"}


def words_size(width, elem):
    return elem * width // words_of(width, elem)


@pytest.mark.parametrize("b,g,nw", [(16384, 16, 16), (1 << 20, 16, 16), (1 << 24, 1, 1), (100, 4096, 2), (1 << 20, 4096, 2),
                                    (1 << 17, 1 << 14, 1), ((1 << 31) - 1, 1, 1)])
def test_rows_of_a_thread_and_the_grid(rule, b, g, nw):  # noqa: F811
    s = rule(b, 1, g, nw, 1)
    assert s["lanes"] * g * s["team"] <= 1 << 31
    assert -(-b // s["lanes"]) <= 64 or s["lanes"] * g * s["team"] * 2 > 1 << 30
