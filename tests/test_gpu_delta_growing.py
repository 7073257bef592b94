"""GPU: decays above 0, by which a matrix grows: the gradient is that of the forward pass, not of one that stops at a
factor of one.  32 steps grow by at most exp(1.6); tolerances as in test_gpu_delta.py (errors grow no faster than what
they are measured by)."""
import pytest
import torch

from test_gpu_delta import BF16, F32, both_passes, check, inputs, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(2, 60, 1, 2, 24, 20), (1, 32, 2, 2, 64, 40)])
def test_both_passes_with_decays_above_0(shape, dtype):
    i = inputs(*shape, dtype, 31)
    gen = torch.Generator(device="cuda").manual_seed(5)
    i["decay"] = 0.1 * torch.rand(i["decay"].shape, generator=gen, device="cuda") - 0.05
    want = reference(i)
    for name, x in both_passes(i).items():
        check(x, want[name], name, want["sizes"].get(name))
