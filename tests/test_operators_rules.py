"""Which variants the operators' rules choose, without a GPU: the GPU tests' shapes reach every instance that a call
can reach, so a changed rule fails here and not by leaving one untested."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1805_11144_amd", "csrc")

SHIM = r'''
#include "operators_rules.hpp"
using namespace ms;
extern "C" {
void sort_rule(int64_t n, int64_t vocab, int64_t* out) {
  int key;
  out[0] = sort_small_items(n), out[1] = sort_bits(vocab, &key), out[2] = sort_items(n), out[3] = sort_tiles(n) > kSortAll;
  out[4] = key;
}
void gated_rule(int64_t batch, int64_t steps, int64_t nv, int64_t* out) {
  const GatedShape s = gated_shape(batch, (steps + kKeep - 1) / kKeep, nv);
  out[0] = s.threads, out[1] = s.nchunk, out[2] = s.groups, out[3] = s.link, out[4] = s.span;
}
void orth_rule(int64_t batch, int64_t rows, int64_t cols, int64_t* out) {
  const OrthShape s = orth_shape(batch, std::min(rows, cols), std::max(rows, cols));
  for (int k = 0; k < 2; ++k) {
    const int64_t c = k ? s.mp : s.np;
    const OrthTile tile = orth_choose(s.pad, k == 0, batch, s.np, c, nullptr);
    out[2 * k] = 64 << tile, out[2 * k + 1] = orth_tiles(tile, k == 0, batch, s.np, c).over > 0;
  }
  out[4] = s.split, out[5] = s.np != std::min(rows, cols);
}
}
'''


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Wextra", "-Werror", "-I", CSRC,
                    str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    lib = C.CDLL(str(d / "shim.so"))

    def call(name, *args):
        out = (C.c_int64 * 6)()
        getattr(lib, name)(*[C.c_int64(a) for a in args], out)
        return list(out)
    return call


def test_sort(rules):
    """(one workgroup's items, or 0; bits of a digit; items; prefix launches)"""
    seen = {tuple(rules("sort_rule", n, v)[:4]) for n, v in [
        (20000, 1000), (20000, 300000), (20000, 100000), (20000, 3000), (131072, 300000), (131073, 65535), (140001, 65536),
        (140001, 200), (300000, 1000), (300000, 3000000), (524289, 65537), (600001, 300000), (600001, 1000), (600001, 250),
        (1048600, 100000)]}
    many = {tuple(rules("sort_rule", n, v)[:4]) for n, v in [
        (1 << 20, 1000), ((1 << 20) + 1, 300000), (1100000, 60000), (3000000, 1000), ((1 << 22) + 77, 300000),
        (5000000, 3000000)]}
    assert {s[1:3] for s in seen if s[0] == 0 and not s[3]} == {(b, i) for b in (8, 9, 10) for i in (4, 8, 16)}
    assert {s[1:3] for s in many | seen if s[3]} == {(8, 16), (9, 16), (10, 16)}
    for n, want in ((1, 1), (1024, 1), (1025, 4), (4096, 4), (4097, 0)):
        assert rules("sort_rule", n, 1000)[0] == want
    for vocab in [1, 2, 255, 256, 1023, 1024, 65535, 65536, (1 << 18) - 1, 1 << 18, (1 << 20) - 1, 1 << 20, (1 << 31) - 1]:
        _, bits, _, _, key = rules("sort_rule", 5000, vocab)[:5]
        assert 8 <= bits <= 10 and key == vocab.bit_length()   # a key may be the vocabulary itself


def test_gated(rules):
    """Chunks in order (three and four of them, in more than 64 workgroups each) and side by side, a wavefront in one
    row and lanes over rows, for one channel and two to a lane."""
    def shape(b, t, d, half):
        return rules("gated_rule", b, t, d // 2 if half and d % 2 == 0 else d)
    for half in (False, True):
        in_order = [shape(*s, half) for s in [(9, 512, 1024), (9, 300, 1024), (90, 400, 130), (90, 385, 96), (150, 500, 60)]]
        assert all(not s[3] and s[2] > 64 for s in in_order)
        assert {(s[1], s[4]) for s in in_order} >= {(3, 0), (4, 0), (4, 1)}
        side = [shape(*s, half) for s in [(2, 3000, 130), (1, 2113, 257), (70, 600, 31), (40, 1700, 1024)]]
        assert all(s[3] and s[1] > 4 for s in side) and {s[4] for s in side} == {0, 1} and max(s[1] for s in side) > 16
    threads, chunks, groups, link, span = shape((1 << 23) + 5, 65, 53, True)[:5]
    assert threads * groups >= 1 << 32 and (chunks, link, span) == (1, 0, 0)


def test_orthogonalised(rules):
    """(tile of X X' and A A, whether its last ones are in quarters, tile of Q X, the same, shares of a sum, padding)"""
    def shape(*s):
        return tuple(rules("orth_rule", *s))
    assert shape(1, 1500, 1500)[:4] == (64, 0, 128, 0)
    assert shape(1, 2900, 2950)[:4] == (128, 1, 128, 1)
    assert shape(8, 1000, 900)[:4] == (128, 1, 128, 0)
    assert shape(1, 3300, 3300)[:4] == (128, 1, 256, 0)
    assert shape(1, 4100, 4000)[:4] == (128, 1, 256, 1)
    assert shape(1, 4096, 4096) == (128, 1, 256, 0, 1, 0)
    assert shape(1, 8192, 8192)[:4] == (256, 1, 256, 0)
    assert shape(1, 520, 600)[:4] == (64, 0, 64, 0) and shape(1, 4100, 4000)[5]
    assert shape(1, 16, 9000)[4] > 1 and shape(1, 600, 600)[4] == 1
