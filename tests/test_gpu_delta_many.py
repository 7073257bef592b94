"""GPU: the gradient of the gated delta rule where its last kernel's workgroups, at most 256, go from chunk to chunk: more
chunks than workgroups, chunks without steps at the start, in the middle and at the end of what a workgroup goes through,
heads that share keys and heads that do not.  Tolerances as in test_gpu_delta.py."""
import numpy as np
import pytest
import torch

from test_gpu_delta import BF16, F32, both_passes, check, inputs, reference

pytestmark = pytest.mark.gpu
CUS = 256


def chunks(dtype, batch, steps, key_heads):
    return batch * key_heads * -(-steps // (64 if dtype == BF16 else 32))


def compared(i):
    want = reference(i, 0.7)
    for name, x in both_passes(i, 0.7).items():
        check(x, want[name], name, want["sizes"].get(name))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(200, 130, 2, 4, 16, 40), (300, 70, 2, 2, 40, 16), (130, 65, 3, 6, 20, 70),
                                   (40, 130, 4, 4, 72, 24)])
def test_more_chunks_than_workgroups(shape, dtype):
    assert chunks(dtype, *shape[:3]) > CUS
    compared(inputs(*shape, dtype, 41, packed=True))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(200, 130, 2, 4, 16, 40), (300, 70, 2, 2, 40, 16)])
@pytest.mark.parametrize("kind", ["any", "many empty", "first empty", "last empty", "only one", "none"])
def test_chunks_without_steps(kind, shape, dtype):
    i = inputs(*shape, dtype, 42)
    batch, steps = shape[:2]
    assert chunks(dtype, *shape[:3]) > CUS
    r = np.random.default_rng(7)
    n = r.integers(0, steps + 1, batch)
    if kind == "many empty":
        n[r.random(batch) < 0.8] = 0
    elif kind == "first empty":   # the first chunks of every workgroup, and more
        n[:batch * 2 // 3] = 0
    elif kind == "last empty":
        n[batch // 3:] = 0
    elif kind == "only one":
        n[:] = 0
        n[batch // 2] = steps
    elif kind == "none":
        n[:] = 0
    i["lengths"] = torch.from_numpy(n).to(torch.int32).to("cuda")
    # dirty memory where results will lie: what is not written shows
    torch.full((sum(x.numel() for x in i.values() if x is not None),), float("nan"), device="cuda")
    compared(i)
