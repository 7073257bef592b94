"""GPU: the decays' gradient of sequences packed into one row.  A sequence takes nothing of the one behind it, not its
rounding either: its bound goes by the sizes of its own states and gradients, however large the next one's values are.

The tolerance is that of test_gpu_delta.py, 4e-5 of the largest |H| |S| (sum over a head's matrix), here of one sequence
and head in place of a row and head."""
import numpy as np
import pytest
import torch

import paper_1805_11144_amd as M
from test_gpu_delta import BF16, F32, TOL, both_passes, inputs, reference

pytestmark = pytest.mark.gpu

NOTHING = [-np.inf, -np.finfo(np.float32).max, -201.0, -150.0, -110.0, -90.0]   # a = 0 in 32 bits


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("factor", [1, 30, 1e3, 1e5])
def test_a_sequence_takes_nothing_of_the_next_ones_rounding(factor, dtype):
    starts = [0, 7, 20, 29, 30, 50, 63, 64, 90, 131]   # of sequences, in steps, in one chunk or another
    steps = 150
    i = inputs(2, steps, 2, 4, 40, 48, dtype, 21)
    for n, s in enumerate(starts[1:]):
        i["decay"][:, s] = float(NOTHING[n % len(NOTHING)])
        if n % 2 == 0:
            i["v"][:, s:starts[n + 2] if n + 2 < len(starts) else steps] *= factor
    want, got = reference(i), both_passes(i)
    g, size = got["ddecay"].double().cpu(), want["sizes"]["ddecay"]
    assert torch.isfinite(g).all()
    for s, e in zip(starts, starts[1:] + [steps]):
        bound = TOL["ddecay"] * size[:, s:e].amax(1, keepdim=True)
        err = (g - want["ddecay"])[:, s:e].abs()
        assert (err <= bound).all(), (s, e, float((err / bound).max()))
        if s:
            assert (g[:, s] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sequences_packed_or_by_themselves(dtype):
    """What each of two sequences learns in a row of both is what it learns in a row of its own, to the roundings of
    sums in other places of a chunk."""
    i = inputs(1, 100, 1, 2, 32, 32, dtype, 22)
    cut = 45
    i["decay"][:, cut] = -float("inf")
    i["v"][:, cut:] *= 1000
    i["dlast"][:] = 0   # of the second one; the first one has none either
    args = [i[n] for n in ("q", "k", "v", "decay", "rate")]
    both = both_passes(i)["ddecay"]
    for part, s0 in ((slice(0, cut), i["s0"]), (slice(cut, 100), None)):
        one = [x[:, part].contiguous() for x in args]
        kept = M.gated_delta(*one, s0=s0, keep=True)[2]
        alone = M.gated_delta_grad(*one, kept, i["dy"][:, part].contiguous())[3]
        want = reference(dict(i, s0=s0 if s0 is not None else None, dlast=None, **{n: i[n][:, part] for n in (
            "q", "k", "v", "decay", "rate", "dy")}))
        bound = 2 * TOL["ddecay"] * want["sizes"]["ddecay"].amax((0, 1))
        assert ((both[:, part] - alone).double().cpu().abs() <= bound).all()
