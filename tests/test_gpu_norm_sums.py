"""GPU: sums of dweight and dbias over many rows and positions of one thread.

dy is one number, 1 + 0.49 * 2^-m, whose tail is lost by every addition to a sum between 2^(23 - m) and 2^(24 - m): a sum of
2048 such numbers one after the other is off by 500 u (u = 2^-24).  In pieces of 64 at most, joined in 64 bits, by 32
rows side by side or by at most 16 one after the other, it is off by at most 64 + 2 * 21 + 4 = 110 u of the sum of sizes
(a piece, two steps of the join with 16 additions and a tree of 5 each, roundings in between)."""
import pytest
import torch

import paper_1805_11144_amd as M

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("batch,positions,groups,width", [
    (1024, 2048, 256, 1),      # by runs: a thread to a channel, one run to a row
    (1100, 2000, 3, 85),
    (16384, 1, 16384, 1),      # by teams: eight rows side by side
    (40000, 1, 2048, 4)])
def test_sums_of_one_number(batch, positions, groups, width):
    channels = groups * width
    x = torch.randn(batch, positions, channels, device="cuda")
    dy = torch.full_like(x, 1 + 0.49 * 2.0 ** -13)
    weight, bias = torch.ones(channels, device="cuda"), torch.zeros(channels, device="cuda")
    _, kept = M.group_norm(x, groups, weight=weight, bias=bias, keep=True)
    _, dweight, dbias = M.group_norm_grad(x, groups, kept, dy, weight=weight, bias=bias)
    n = batch * positions
    want = n * float(dy[0, 0, 0].double())
    assert float((dbias.double() - want).abs().max()) <= 110 * U * want
    # dweight: the normalised values' sum, from the same mean and deviation in 64 bits
    exact, size = (torch.zeros(channels, dtype=torch.float64, device="cuda") for _ in range(2))
    for rows in range(0, batch, 256):
        part = slice(rows, rows + 256)
        mean, rstd = kept[part].double().unbind(-1)
        h = (x[part].double().view(-1, positions, groups, width) - mean[:, None, :, None]) * rstd[:, None, :, None]
        exact += h.sum((0, 1)).reshape(-1) * dy[0, 0, 0].double()
        size += h.abs().sum((0, 1)).reshape(-1) * dy[0, 0, 0].double()
    # a value's own: its difference from the mean and two products, 4 u, which add up at random and are a piece's 64 at most
    assert ((dweight.double() - exact).abs() <= 110 * U * size + 1e-30).all()
