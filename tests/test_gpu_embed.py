"""GPU: table lookup and its gradient against 64 bits.

Tolerances: a looked-up row is one 32-bit product rounded once, so it equals torch's bit for bit.  A gradient
row is a 32-bit sum of L rows times the scale: its error is at most (L + 2) 2^-24 times the sum of the terms'
sizes, plus half a unit of the result's type."""
import numpy as np
import pytest
import torch

import paper_1805_11144_amd as M

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def inputs(n, vocab, dim, dtype, ids, seed, skew=False):
    r = np.random.default_rng([seed, n, vocab, dim])
    t = (np.exp(r.uniform(0, np.log(vocab + 1), n)) - 1).astype(np.int64) if skew else r.integers(0, vocab, n)
    t = np.minimum(t, vocab - 1)
    t[r.random(n) < 0.1] = -1
    if n > 3:
        t[1], t[2] = vocab, np.iinfo(np.int32).min   # outside the table on either side
    if n > 4 and ids == torch.int64:
        t[3] = (1 << 32) + 1                          # its low half is a token of the table
    table = torch.from_numpy(r.standard_normal((vocab, dim))).to(dtype).to(DEV)
    rows = torch.from_numpy(r.standard_normal((n, dim))).to(dtype).to(DEV)
    return torch.from_numpy(t).to(ids).to(DEV), table, rows


def grad64(tokens, rows, vocab, scale):
    """(gradient, sum of sizes, count) in 64 bits on the host."""
    t, x = tokens.cpu().numpy().astype(np.int64).ravel(), rows.double().cpu().numpy().reshape(-1, rows.shape[-1])
    live = (t >= 0) & (t < vocab)
    g, s = np.zeros((vocab, x.shape[1])), np.zeros((vocab, x.shape[1]))
    np.add.at(g, t[live], x[live])
    np.add.at(s, t[live], np.abs(x[live]))
    return g * scale, s * abs(scale), np.bincount(t[live], minlength=vocab)[:, None]


def check_grad(got, tokens, rows, scale, before=None):
    want, size, count = grad64(tokens, rows, got.shape[0], scale)
    if before is not None:
        want, size = want + before, size + np.abs(before)
    half = 2.0 ** (-24 if got.dtype == F32 else -8)   # float32 has 24 significant bits, bf16 has 8
    err = np.abs(got.double().cpu().numpy() - want)
    bound = (count + 2) * 2.0 ** -24 * size * (1 + 2 * half) + half * np.abs(want) * 1.01
    assert (err <= bound).all(), float((err - bound).max())


SHAPES = [(1, 1, 1), (1, 7, 3), (5, 2, 16), (64, 1000, 192), (63, 3, 17), (300, 5000, 333), (1000, 70000, 8),
          (257, 9, 1024), (33, 300, 1500)]


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,vocab,dim", SHAPES)
def test_lookup_and_gradient(n, vocab, dim, dtype, ids):
    tokens, table, rows = inputs(n, vocab, dim, dtype, ids, 1)
    scale = dim ** 0.5
    got = M.embed(tokens, table, scale=scale)
    live = (tokens >= 0) & (tokens < vocab)
    want = (table[torch.where(live, tokens, 0).long()].float() * np.float32(scale)).to(dtype)
    assert torch.equal(got, torch.where(live[:, None], want, torch.zeros_like(want)))
    for gd in (F32, BF16):
        out = torch.full((vocab, dim), float("nan"), dtype=gd, device=DEV)
        check_grad(M.embed_grad(tokens, rows, scale=scale, out=out), tokens, rows, scale)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,vocab,dim", [(4096, 300, 40), (4097, 65535, 24), (20000, 65536, 33), (50000, 1 << 20, 8),
                                         (70001, 17, 96), (30000, 1 << 17, 1)])
def test_gradient_of_many_tokens(n, vocab, dim, dtype):
    """Several tiles of the sort, one to three digits, runs from none to thousands."""
    for skew in (False, True):
        tokens, _, rows = inputs(n, vocab, dim, dtype, torch.int32, 2, skew)
        check_grad(M.embed_grad(tokens, rows, vocab, scale=0.5), tokens, rows, 0.5)


@pytest.mark.parametrize("fill", [0, 5, -1, 9])
def test_one_token_everywhere(fill):
    """All rows in one sum, at the first, a middle and the last row of the table, or in none."""
    n, vocab, dim = 10007, 10, 130
    _, _, rows = inputs(n, vocab, dim, F32, torch.int32, 3)
    tokens = torch.full((n,), fill, dtype=torch.int32, device=DEV)
    check_grad(M.embed_grad(tokens, rows, vocab), tokens, rows, 1.0)


def test_gradient_has_the_same_bits_again():
    tokens, _, rows = inputs(50000, 200, 64, BF16, torch.int64, 4, True)
    first = M.embed_grad(tokens, rows, 200)
    for _ in range(3):
        assert torch.equal(first, M.embed_grad(tokens, rows, 200))


def test_rows_hold_no_trace_of_masked_ones():
    """Infinities and NaN in the rows of padding, and table rows that no token names."""
    tokens, table, rows = inputs(500, 50, 20, F32, torch.int32, 5)
    dead = (tokens < 0) | (tokens >= 50)
    rows[dead] = float("nan")
    check_grad(M.embed_grad(tokens, rows, 50), tokens, torch.where(dead[:, None], 0.0, rows), 1.0)
    tokens = tokens.clamp(max=20)
    table[30:] = float("inf")
    assert torch.isfinite(M.embed(tokens, table)).all()
    # and a NaN that is named stays where it is named
    rows[:] = 1.0
    at = int(torch.nonzero(tokens >= 0)[0])
    rows[at, 3] = float("nan")
    g = M.embed_grad(tokens, rows, 50)
    assert torch.isnan(g[tokens[at], 3]) and torch.isnan(g).sum() == 1


@pytest.mark.parametrize("gd", [F32, BF16])
def test_accumulate(gd):
    tokens, _, rows = inputs(3000, 400, 24, BF16, torch.int64, 6, True)
    out = torch.randn(400, 24, device=DEV).to(gd)
    before = out.double().cpu().numpy()
    got = M.embed_grad(tokens, rows, scale=2.0, out=out, accumulate=True)
    assert got is out
    check_grad(out, tokens, rows, 2.0, before)
    count = grad64(tokens, rows, 400, 1.0)[2][:, 0]
    assert (count == 0).any() and np.array_equal(out.double().cpu().numpy()[count == 0], before[count == 0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset", [0, 1, 2, 4])
def test_strides_and_alignment(dtype, offset):
    """Tables, gradients and rows inside wider arrays, from any element on."""
    vocab, dim, n = 40, 24, 100
    tokens, table, rows = inputs(n, vocab, dim, dtype, torch.int32, 7)
    wide = torch.full((vocab, dim + 9), float("nan"), dtype=dtype, device=DEV)
    wide[:, offset:offset + dim] = table
    view = wide[:, offset:offset + dim]
    assert torch.equal(M.embed(tokens, view, scale=3.0), M.embed(tokens, table, scale=3.0))
    wide_rows = torch.full((n, dim + 9), float("nan"), dtype=dtype, device=DEV)
    wide_rows[:, offset:offset + dim] = rows
    out = torch.full((vocab, dim + 9), 7.0, device=DEV)
    got = M.embed_grad(tokens, wide_rows[:, offset:offset + dim], out=out[:, offset:offset + dim])
    check_grad(got, tokens, rows, 1.0)
    assert (out[:, :offset] == 7).all() and (out[:, offset + dim:] == 7).all()


def test_token_shapes_and_broadcast_rows():
    tokens, table, rows = inputs(60, 30, 16, F32, torch.int64, 8)
    t = tokens.view(3, 4, 5)
    assert torch.equal(M.embed(t, table).view(60, 16), M.embed(tokens, table))
    assert torch.equal(M.embed(t.transpose(0, 2), table), M.embed(t.transpose(0, 2).contiguous(), table))
    one = rows[:1].expand(60, 16)
    check_grad(M.embed_grad(tokens, one, 30), tokens, one.contiguous(), 1.0)
    assert torch.equal(M.embed_grad(t, rows.view(3, 4, 5, 16), 30), M.embed_grad(tokens, rows, 30))


def test_no_tokens():
    tokens = torch.empty(0, dtype=torch.int32, device=DEV)
    assert M.embed(tokens, torch.ones(4, 8, device=DEV)).shape == (0, 8)
    out = torch.full((4, 8), float("nan"), device=DEV)
    M.embed_grad(tokens, torch.empty(0, 8, device=DEV), out=out)
    assert (out == 0).all()
    out.fill_(3.0)
    M.embed_grad(tokens, torch.empty(0, 8, device=DEV), out=out, accumulate=True)
    assert (out == 3).all()


def test_offsets_past_32_bits():
    """A table and its gradient of more than 2^31 values."""
    vocab, dim = 70000, 32768
    table = torch.zeros(vocab, dim, dtype=BF16, device=DEV)
    ids = torch.tensor([vocab - 1, 65537, 0, vocab - 1], device=DEV)
    for v in set(ids.tolist()):
        table[v] = v % 100 + 1
    got = M.embed(ids, table)
    assert torch.equal(got.double(), ((ids % 100 + 1)[:, None].double()).expand(4, dim))
    out = table
    M.embed_grad(ids, got, out=out)
    want = {v: 0.0 for v in set(ids.tolist())}
    for v in ids.tolist():
        want[v] += v % 100 + 1
    for v, x in want.items():
        assert (out[v] == x).all()
    assert (out[1:65537] == 0).all() and (out[65538:-1] == 0).all()


def test_another_stream_and_a_graph():
    tokens, table, rows = inputs(5000, 100, 64, F32, torch.int64, 9, True)
    want, grad = M.embed(tokens, table), M.embed_grad(tokens, rows, 100)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        t, x, r = tokens.clone(), table.clone(), rows.clone()
        a, b = M.embed(t, x), M.embed_grad(t, r, 100)
    side.synchronize()
    assert torch.equal(a, want) and torch.equal(b, grad)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = M.embed(tokens, table), M.embed_grad(tokens, rows, 100)
    for k in range(3):
        table.mul_(-1.0)
        rows.mul_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        sign = -1.0 if k % 2 == 0 else 1.0
        assert torch.equal(a, want * sign) and torch.equal(b, grad * sign)
