"""GPU: orthogonalised updates of matrices whose iterates are small: norms far below eps, where X0 = X / (|X| + eps) is
small, and coefficients that shrink it.

Tolerance (2-norm of the difference over 2-norm of the result): 3.4e-3 as for any spectrum (test_gpu_orth_spectra.py),
and for coefficients that move all singular values of these matrices alike 1e-4, as in test_gpu_orth.py."""
import pytest
import torch

import paper_1805_11144_amd as M
from test_gpu_orth import BF16, DEV, F32, TOL, matrices, off, orth64

pytestmark = pytest.mark.gpu
SHAPES = [(20, 30), (90, 80), (40, 1500), (600, 520), (1100, 1000)]


def sized(batch, rows, cols, sizes, dtype=F32, seed=60):
    x = matrices(batch, rows, cols, seed)
    return (x / torch.linalg.matrix_norm(x)[:, None, None] * torch.tensor(sizes, dtype=torch.float64)[:, None, None]).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [1e-4, 1e-7, 1e-9, 1e-10, 1e-12, 1e-14, 1e-18, 1e-30])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norms_below_eps(rows, cols, size, dtype):
    x = sized(1, rows, cols, [size], dtype)
    assert off(M.orthogonalise(x.to(DEV)), orth64(x)) <= 3.4e-3 + (2.0 ** -8 if dtype == BF16 else 0.0)


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norms_of_a_batch_differ(rows, cols):
    sizes = [1.0, 1e-12, 0.0, 1e-7, 1e-20, 1e5]
    x = sized(6, rows, cols, sizes)
    got, want = M.orthogonalise(x.to(DEV)), orth64(x)
    for k, size in enumerate(sizes):
        if size == 0.0:
            assert (got[k] == 0).all()
        else:
            assert off(got[k], want[k]) <= 3.4e-3, size


@pytest.mark.parametrize("steps,coef", [(3, (1e-3, 0.0, 0.0)), (8, (0.01, 0.0, 0.0)), (1, (1e-9, 0.0, 0.0)),
                                        (10, (0.05, -0.02, 0.01)), (40, (0.5, 0.0, 0.0)), (2, (30.0, 0.0, 0.0))])
@pytest.mark.parametrize("size", [1.0, 1e-10])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_coefficients_that_shrink_or_grow(rows, cols, size, steps, coef):
    x = sized(1, rows, cols, [size])
    assert off(M.orthogonalise(x.to(DEV), steps=steps, coefficients=coef), orth64(x, steps, coef)) <= TOL[F32] * max(1, steps / 5)


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_many_steps_bring_a_small_norm_up(rows, cols):
    """1.5 s - 0.5 s^3 from X0 of norm 1e-8: 60 steps bring the smallest up, the others to singular values of one."""
    x = sized(1, rows, cols, [1e-15])
    got = M.orthogonalise(x.to(DEV), steps=80, coefficients=(1.5, -0.5, 0.0))[0].double()
    gram = got @ got.T if rows <= cols else got.T @ got
    assert float((gram - torch.eye(min(rows, cols), device=DEV)).abs().max()) <= 1e-4


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_update_from_a_small_gradient(rows, cols):
    g = sized(1, rows, cols, [1e-13])[0]
    w, m = torch.zeros(rows, cols, device=DEV), torch.zeros(rows, cols, device=DEV)
    M.orthogonal_update(w, m, g.to(DEV), rate=0.5, nesterov=False)
    assert off(w, -0.5 * orth64(g)) <= 3.4e-3
