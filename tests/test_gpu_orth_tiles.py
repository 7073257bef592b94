"""GPU: orthogonalised updates on every kind of tile: 128 x 128 and 256 x 256, with the last tiles of a launch in
quarters, padded, into results and into weights (that the rule takes these tiles for these shapes is checked
where it can be without a GPU, in test_operators_rules.py).

Matrices are U diag(s) W with dense orthogonal U and W (cosines with random signs) and s within a factor of 20; what
each is compared with are the products in 64 bits.  Tolerances: those of test_gpu_orth.py for such matrices."""
import math

import pytest
import torch

import paper_1805_11144_amd as M
from test_gpu_orth import BF16, DEV, F32, TOL

pytestmark = pytest.mark.gpu
F64 = torch.float64


def cosines(n, gen):
    """A dense orthogonal matrix."""
    i = torch.arange(n, dtype=F64, device=DEV)
    c = torch.cos(math.pi / n * (i[None] + 0.5) * i[:, None]) * math.sqrt(2 / n)
    c[0] *= math.sqrt(0.5)
    return c * (2.0 * torch.randint(2, (n,), generator=gen, device=DEV) - 1)


def matrices(batch, rows, cols, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n, out = min(rows, cols), []
    for _ in range(batch):
        s = torch.exp(-math.log(20) * torch.rand(n, generator=gen, device=DEV, dtype=F64))
        out.append((cosines(rows, gen)[:, torch.randperm(rows, generator=gen, device=DEV)[:n]] * s) @
                   cosines(cols, gen)[torch.randperm(cols, generator=gen, device=DEV)[:n]])
    return torch.stack(out)


def products64(x, coef=M.operators.NEWTON_SCHULZ):
    out = []
    for y in x.double():
        tall = y.shape[0] > y.shape[1]
        y = (y.T if tall else y).contiguous()
        y = y / (torch.linalg.norm(y) + 1e-7)
        for _ in range(5):
            a = y @ y.T.contiguous()
            y = coef[0] * y + (coef[1] * a + coef[2] * (a @ a)) @ y
        out.append(y.T if tall else y)
    return torch.stack(out)


def off(got, want):
    return float(torch.linalg.norm(got.double() - want) / torch.linalg.norm(want))


SHAPES = [(1, 1500, 1500), (1, 2900, 2950), (8, 1000, 900), (1, 3300, 3300), (1, 4100, 4000)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,rows,cols", SHAPES)
def test_results(batch, rows, cols, dtype):
    x = matrices(batch, rows, cols, 1).to(dtype)
    got = M.orthogonalise(x)
    assert off(got, products64(x)) <= TOL[dtype]
    assert torch.equal(got, M.orthogonalise(x))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,rows,cols", SHAPES)
def test_updates(batch, rows, cols, dtype):
    g = matrices(batch, rows, cols, 2).to(dtype)
    w0 = matrices(batch, rows, cols, 3)
    w, m = w0.float(), torch.zeros(batch, rows, cols, device=DEV)
    M.orthogonal_update(w, m, g, rate=0.5, weight_decay=0.1, nesterov=False)
    assert torch.equal(m, g.float())
    assert off(w, 0.95 * w0 - 0.5 * products64(g)) <= TOL[F32]


def test_symmetric_products_on_the_largest_tiles():
    """8192 x 8192: X X' and A A take 256 x 256 tiles too, the last ones in quarters."""
    x = matrices(1, 8192, 8192, 4).to(F32)
    assert off(M.orthogonalise(x), products64(x)) <= TOL[F32]
