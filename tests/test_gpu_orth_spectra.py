"""GPU: orthogonalised updates of matrices whose singular values are spread as a gradient's are: a few strong
directions over small noise, low rank, a power law.

Tolerances (2-norm of the difference over 2-norm of the result).  A step's four roundings (X, A, Q and the sums)
are 2^-22 of their values' sizes, and what they leave grows like a small singular value, by at most 3.4445^5 = 485
over the five steps, while the iterate itself ends no smaller than 0.7 of its largest norm: 5 * 4 * 485 * 2^-22 / 0.7
= 3.4e-3.  A bf16 result adds half a unit of its own, 2^-8."""
import numpy as np
import pytest
import torch

import paper_1805_11144_amd as M
from test_gpu_orth import BF16, DEV, F32, off, orth64

pytestmark = pytest.mark.gpu
TOL = {F32: 3.4e-3, BF16: 3.4e-3 + 2.0 ** -8}


def spectrum(kind, rows, cols):
    r = np.random.default_rng([50, rows, cols])
    strong = r.standard_normal((rows, 16)) @ r.standard_normal((16, cols)) / 4
    noise = r.standard_normal((rows, cols))
    if kind == "power":
        n = min(rows, cols)
        u, _, w = np.linalg.svd(noise, full_matrices=False)
        x = (u * (1 + np.arange(n)) ** -1.5) @ w
    else:
        x = strong + {"rank 16": 0.0, "0.1%": 1e-3, "1%": 1e-2}[kind] * noise
    return torch.from_numpy(1e-3 * x)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["rank 16", "0.1%", "1%", "power"])
@pytest.mark.parametrize("rows,cols", [(768, 800), (1024, 1024), (1100, 900), (300, 200), (40, 100)])
def test_wide_spectra(rows, cols, kind, dtype):
    x = spectrum(kind, rows, cols).to(dtype)
    assert off(M.orthogonalise(x.to(DEV)), orth64(x)) <= TOL[dtype]


@pytest.mark.parametrize("kind", ["rank 16", "1%", "power"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_update_of_wide_spectra(kind, dtype):
    g = spectrum(kind, 900, 1000).to(dtype)
    w, m = torch.zeros(900, 1000, device=DEV), torch.zeros(900, 1000, device=DEV)
    M.orthogonal_update(w, m, g.to(DEV), rate=0.5, nesterov=False)
    assert torch.equal(m, g.to(DEV).float())
    assert off(w, -0.5 * orth64(g)) <= TOL[F32]
