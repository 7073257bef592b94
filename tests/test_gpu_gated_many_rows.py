"""GPU: the gated lowpass of more rows than one grid holds workgroups for: 2^23 + 5 rows of 65 steps, which take
eight wavefronts each, 2^32 threads.  Rows at both ends, and around where a grid's 2^31 threads end, have the bits
that they have in a call of their own."""
import pytest
import torch

import paper_1805_11144_amd as M

pytestmark = pytest.mark.gpu
DEV, BF16 = "cuda", torch.bfloat16
B, T, D = (1 << 23) + 5, 65, 53


def test_more_rows_than_a_grid_holds():
    gen = torch.Generator(device=DEV).manual_seed(0)
    v, g, dy = (torch.randn(B, 1, D, generator=gen, device=DEV, dtype=BF16) for _ in range(3))
    at = torch.tensor([0, 1, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, (1 << 23) - 1, 1 << 23, B - 2, B - 1], device=DEV)
    few = [x[at].expand(-1, T, D) for x in (v, g, dy)]
    many = [x.expand(B, T, D) for x in (v, g, dy)]
    want, last, kept = M.gated_lowpass(few[0], few[1], keep=True)
    dv, dg, dy0 = M.gated_lowpass_grad(few[0], few[1], kept, few[2])
    y, end, kept = M.gated_lowpass(many[0], many[1], keep=True)
    assert torch.equal(y[at], want) and torch.equal(end[at], last)
    del y, end
    got = M.gated_lowpass_grad(many[0], many[1], kept, many[2])
    assert all(torch.equal(x[at], w) for x, w in zip(got, (dv, dg, dy0)))
