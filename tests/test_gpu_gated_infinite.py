"""GPU: infinities and NaN in the gated lowpass.  Joined runs of steps give what single steps give: an infinite state
stays infinite under any gate above 0, however small the product of the gates; a gate of 0 (g = -inf) takes nothing
of the state, and one of 1 (g = +inf) nothing of the input, whatever they are, in both directions."""
import math

import pytest
import torch

import paper_1805_11144_amd as M
from test_gpu_gated import BF16, DEV, F32, both_passes, check, inputs, reference

pytestmark = pytest.mark.gpu
BAD = (math.nan, math.inf, -math.inf)
SHAPES = [(1, 20), (2, 100), (2, 300), (150, 500), (1, 3000)]   # one run, one chunk, several in order, side by side


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("gate", [-3.0, -8.0, -60.0])
@pytest.mark.parametrize("b,t", SHAPES)
def test_infinite_states_stay_infinite(b, t, gate, dtype):
    d = 66
    v, g, y0, _, dy, dlast = inputs(b, t, d, dtype, 20)
    g = torch.full_like(g, gate)
    want = reference(v, g, y0, None, dy, dlast)
    y0[:, 0], y0[:, 1], y0[:, 2] = math.inf, -math.inf, math.inf
    dlast[:, 2:5] = torch.tensor([math.inf, math.inf, -math.inf], device=DEV)
    got = both_passes(v, g, y0, None, dy, dlast)
    for c, s in ((0, math.inf), (1, -math.inf), (2, math.inf)):
        assert (got["y"][:, :, c] == s).all() and (got["last"][:, c] == s).all()
        assert torch.isinf(got["dg"][:, :, c]).all()
    for c, s in ((2, math.inf), (3, math.inf), (4, -math.inf)):
        assert (got["dv"][:, :, c] == s).all() and (got["dy0"][:, c] == s).all()
        # y[t-1] - v[t] can be 0 where a value comes twice under a nearly closed gate: 0 times infinity
        once = torch.ones(b, t, dtype=torch.bool, device=DEV)
        once[:, 1:] = v[:, 1:, c] != v[:, :-1, c]
        assert torch.isinf(got["dg"][:, :, c][once]).all()
    rest = {"y": slice(3, None), "last": slice(3, None), "dv": slice(5, None), "dg": slice(5, None), "dy0": slice(5, None)}
    for name, x in got.items():
        value, bound = want[name]
        check(x[..., rest[name]], (value[..., rest[name]], bound[..., rest[name]]), name)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t", SHAPES)
def test_a_packed_sequence_keeps_its_values_to_itself(b, t, dtype):
    """NaN and infinities in one sequence of a packed row, in the state before it and in the gradient behind it."""
    d = 66
    v, g, y0, _, dy, dlast = inputs(b, t, d, dtype, 21)
    starts = [s for s in (0, 7, 16, 37, 90, 128, 300, 417, 1029, 2048) if s < t]
    g[:, starts] = -math.inf
    edges = starts + [t]
    clean = both_passes(v, g, y0, None, dy, dlast)
    for k in range(len(starts)):
        lo, hi = edges[k], edges[k + 1]
        for bad in BAD:
            w, z, h, e = v.clone(), dy.clone(), y0.clone(), dlast.clone()
            w[:, lo:hi, 1::3] = bad
            z[:, lo:hi, 2::3] = bad
            h[:] = bad
            if hi == t:
                e[:] = bad
            y, last, kept = M.gated_lowpass(w, g, y0=h, keep=True)
            dv, dg, dy0 = M.gated_lowpass_grad(w, g, kept, z, dlast=e)
            got = dict(y=y, last=last, dv=dv, dg=dg, dy0=dy0)
            other = torch.ones(t, dtype=torch.bool, device=DEV)
            other[lo:hi] = False
            for name in ("y", "dv", "dg"):
                assert torch.equal(got[name][:, other], clean[name][:, other]), (name, lo, bad)
            if hi < t:
                assert torch.equal(got["last"], clean["last"])
            assert (got["dy0"] == 0).all()
            assert not torch.isfinite(got["y"][:, lo:hi, 1::3]).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t", SHAPES)
def test_an_open_gate_takes_nothing_of_its_input(b, t, dtype):
    d = 66
    v, g, y0, _, dy, dlast = inputs(b, t, d, dtype, 22)
    held = torch.rand(b, t, device=DEV) < 0.3
    g[held] = math.inf
    clean = both_passes(v, g, y0, None, dy, dlast)
    for bad in BAD:
        w = v.clone()
        w[held] = bad
        for name, x in both_passes(w, g, y0, None, dy, dlast).items():
            assert torch.equal(x, clean[name]), (name, bad)
    g[:] = math.inf
    dlast[:] = math.inf
    got = both_passes(v, g, y0, None, dy, dlast)
    assert (got["dv"] == 0).all() and (got["dg"] == 0).all() and (got["dy0"] == math.inf).all()


@pytest.mark.parametrize("bad", BAD)
def test_single_steps(bad):
    state = torch.full((3, 5), bad, device=DEV)
    v, g = torch.randn(3, 5, device=DEV), torch.zeros(3, 5, device=DEV)
    g[0] = -math.inf
    y = M.gated_lowpass_step(v, g, state)
    assert torch.equal(y[0], v[0]) and torch.equal(state[0], v[0]) and not torch.isfinite(state[1:]).any()
    state = torch.randn(3, 5, device=DEV)
    before = state.clone()
    y = M.gated_lowpass_step(torch.full_like(v, bad), torch.full_like(g, math.inf), state)
    assert torch.equal(y, before) and torch.equal(state, before)
