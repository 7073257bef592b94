"""GPU: orthogonalised updates of matrices whose norm is far below eps: X0 = X / (|X| + eps) is small, and the tiled
kernels hold its values in steps of 2^-38 (16-bit parts end at 2^-24, scaled by 2^14), the one-workgroup kernel in 32
bits.

Tolerances (2-norm): 3.4e-3 of the result as for any spectrum (test_gpu_orth_spectra.py), and for the tiled kernels
half a step for each of the n m values at each of the five iterates, which grows by 3.4445 in each that follows:
sqrt(n m) 2^-39 (485 + 141 + 41 + 12 + 3)."""
import math

import pytest
import torch

import paper_1805_11144_amd as M
from test_gpu_orth import DEV, matrices, orth64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [1e-7, 1e-10, 1e-12, 1e-14, 1e-18])
@pytest.mark.parametrize("rows,cols", [(20, 30), (90, 80), (600, 520)])
def test_norms_below_eps(rows, cols, size):
    x = matrices(1, rows, cols, 60).float()
    x = x * (size / float(torch.linalg.norm(x)))
    got, want = M.orthogonalise(x.to(DEV)).double().cpu(), orth64(x)
    step = 0.0 if min(rows, cols) <= 64 else math.sqrt(rows * cols) * 2.0 ** -39 * 682
    assert torch.isfinite(got).all()
    assert float(torch.linalg.norm(got - want)) <= 3.4e-3 * float(torch.linalg.norm(want)) + step
