"""GPU: silu in group norm, relative to itself.  A weight of 0 makes the bias the activation's argument, exactly.

In units u = 2^-24: 1 / (1 + exp(-z)) takes exp (2 u of the argument's product, split in two, and 2 u of its own), a
sum (1 u) and a reciprocal (2 u), silu one product more: 8 u = 4.8e-7 of silu(z) for every z whose exponential is finite
in 32 bits.  The derivative g (1 + z (1 - g)) is good to as much of g (1 + |z|): 1 - g has g's error.  The hardware's
reciprocal is 0 where it would be below 2^-126, the smallest normal number; that is from |z| = 87.3 on, and exp(-z) is
infinite from 88.8 on, so silu and its derivative lose 89 * 2^-126 at most."""
import numpy as np
import pytest
import torch

import paper_1805_11144_amd as M

pytestmark = pytest.mark.gpu
TINY = 89 * 2.0 ** -126


def arguments():
    z = np.concatenate([np.linspace(-90, 30, 3001), -np.logspace(-6, 1.9, 800), np.logspace(-6, 38, 295)])
    return torch.from_numpy(z).float()


@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("positions", [1, 40])   # by teams, and by runs
def test_relative_errors(positions, rows):
    z = arguments()
    c = z.numel()
    x = torch.randn(rows, positions, c, device="cuda")
    w = dict(weight=torch.zeros(c, device="cuda"), bias=z.cuda(), activation="silu")
    y, kept = M.group_norm(x, 8, **w, keep=True)
    exact = z.double()
    g = torch.sigmoid(exact)
    want = exact * g
    err = (y.double().cpu() - want).abs()
    assert (err <= 8 * 2.0 ** -24 * want.abs() + TINY).all(), float((err / (want.abs() + TINY)).max())
    dy = torch.zeros_like(x)
    dy[rows // 2, positions // 2] = 1.0   # dbias is one value's derivative
    dx, _, dbias = M.group_norm_grad(x, 8, kept, dy, **w)
    assert (dx == 0).all()
    want = g * (1 + exact * (1 - g))
    err = (dbias.double().cpu() - want).abs()
    bound = 8 * 2.0 ** -24 * g * (1 + exact.abs()) + TINY
    assert (err <= bound).all(), float((err / bound).max())


def plain(z, act):
    return {"none": z, "relu": torch.where(z > 0, z, torch.where(z != z, z, 0.0)), "silu": z / (1 + torch.exp(-z))}[act]


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("positions", [1, 40])
def test_arguments_that_are_infinite_or_no_numbers(positions, act):
    """z as the bias sets it: results are what the activation's definition gives in 32 bits, and others' stay."""
    inf, nan = float("inf"), float("nan")
    bias = torch.tensor([inf, -inf, nan, 3e38, -3e38, 1e30, -1e30, 200.0, -200.0, -100.0, 89.0, 0.0, -0.0, 1.0, -1.0, 0.5])
    c = bias.numel()
    x = torch.randn(5, positions, c, device="cuda")
    w = dict(weight=torch.zeros(c, device="cuda"), activation=act)
    y, kept = M.group_norm(x, 2, bias=bias.cuda(), **w, keep=True)
    want = plain(bias, act).expand(y.shape)
    got = y.cpu()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
    fine = want.isfinite()
    assert torch.allclose(got[fine], want[fine], rtol=1e-6, atol=1e-37)
    assert torch.equal(got[want == inf], want[want == inf]) and torch.equal(got[want == -inf], want[want == -inf])
    fine = bias.isfinite()
    dx, dweight, dbias = M.group_norm_grad(x, 2, kept, torch.ones_like(x), bias=bias.cuda(), **w)
    assert torch.isfinite(dbias.cpu()[fine]).all() and torch.isfinite(dweight.cpu()[fine]).all()


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("shape", [(6, 1, 4, 24), (6, 40, 4, 24), (4, 700, 3, 40)])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_a_group_that_holds_an_infinity_or_nan_keeps_it(bad, shape, act):
    b, t, g, width = shape
    x, dy = torch.randn(b, t, g * width, device="cuda"), torch.randn(b, t, g * width, device="cuda")
    w = dict(weight=torch.randn(g * width, device="cuda"), bias=torch.randn(g * width, device="cuda"), activation=act)

    def all_of(x):
        y, kept = M.group_norm(x, g, **w, keep=True)
        dx, dweight, dbias = M.group_norm_grad(x, g, kept, dy, **w)
        parts = lambda a: a.view(b, t, g, width)  # noqa: E731
        return parts(y), parts(dx), dweight.view(g, width), dbias.view(g, width)
    want = all_of(x)
    x = x.clone()
    x[1, t // 2, width + 3] = bad   # row 1, group 1
    y, dx, dweight, dbias = all_of(x)
    others = torch.ones(b, g, dtype=torch.bool, device="cuda")
    others[1, 1] = False
    for got, ref in ((y, want[0]), (dx, want[1])):
        assert torch.equal(got.transpose(1, 2)[others], ref.transpose(1, 2)[others])
        assert got[1, :, 1].isnan().all()
    keep = torch.arange(g, device="cuda") != 1
    assert torch.equal(dweight[keep], want[2][keep]) and torch.equal(dbias[keep], want[3][keep])
