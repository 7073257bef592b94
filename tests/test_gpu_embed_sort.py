"""GPU: the table's gradient over every size of digit and of tile of its sort, on either side of where they change.
Tolerances: those of test_gpu_embed.py."""
import pytest
import torch

import paper_1805_11144_amd as M
from test_gpu_embed import BF16, DEV, F32, check_grad, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("skew", [False, True])
@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,vocab", [
    (20000, 1000), (20000, 300000), (20000, 100000), (20000, 3000), (131072, 300000), (131073, 65535), (140001, 65536),
    (140001, 200), (300000, 1000), (300000, 3000000), (524289, 65537), (600001, 300000), (600001, 1000), (600001, 250),
    (1048600, 100000)])
def test_digits_and_tiles(n, vocab, ids, skew):
    tokens, _, rows = inputs(n, vocab, 3, F32, ids, 10, skew)
    got = M.embed_grad(tokens, rows, vocab, scale=0.5)
    check_grad(got, tokens, rows, 0.5)
    assert torch.equal(got, M.embed_grad(tokens, rows, vocab, scale=0.5))


def test_tokens_in_descending_order():
    """No two pairs stay where they are; runs of one, in tiles that end inside a wavefront."""
    n = 600001
    tokens = torch.arange(n - 1, -1, -1, dtype=torch.int32, device=DEV)
    rows = torch.arange(n, dtype=F32, device=DEV)[:, None].contiguous()
    assert torch.equal(M.embed_grad(tokens, rows, n), rows.flip(0))
