"""GPU: the gated lowpass with three and four chunks of a row gone through by one workgroup, in many workgroups, where
each chunk takes its state from the one before and the wavefronts' maps use their two places in turn.  Tolerances:
those of test_gpu_gated.py."""
import pytest
import torch

from test_gpu_gated import BF16, F32, both_passes, check, inputs, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("packed,ragged", [(False, False), (True, True)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t,d", [(9, 512, 1024), (9, 300, 1024), (90, 400, 130), (90, 385, 96), (150, 500, 60)])
def test_chunks_in_order(b, t, d, dtype, packed, ragged):
    v, g, y0, lengths, dy, dlast = inputs(b, t, d, dtype, 17, packed, ragged)
    want = reference(v, g, y0, lengths, dy, dlast)
    got = both_passes(v, g, y0, lengths, dy, dlast)
    for name, x in got.items():
        check(x, want[name], name)
    again = both_passes(v, g, y0, lengths, dy, dlast)
    assert all(torch.equal(got[k], again[k]) for k in got)
