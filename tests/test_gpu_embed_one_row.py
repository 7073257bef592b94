"""GPU: the table's gradient of a single token whose row has strides of its own, as of several such rows."""
import pytest
import torch

import paper_1805_11144_amd as M
from test_gpu_embed import DEV, check_grad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 2])
def test_rows_with_strides(n):
    tokens = torch.arange(n, device=DEV)
    x = torch.randn(n, 24, device=DEV)
    for rows in (x[:, ::2], x[:, :1].expand(n, 12), x[:1, :1].expand(n, 12), x.T.contiguous().T[:, :12]):
        check_grad(M.embed_grad(tokens, rows, 3), tokens, rows.contiguous(), 1.0)
