"""GPU: the table's gradient of millions of tokens: right, and in a time that grows as they do."""
import numpy as np
import pytest
import torch

import paper_1805_11144_amd as M
from test_gpu_embed import DEV

pytestmark = pytest.mark.gpu


def case(n, vocab, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    tokens = torch.randint(-1, vocab + 1, (n,), generator=gen, device=DEV, dtype=torch.int32)
    # whole numbers whose sums float32 holds exactly, in any order
    return tokens, torch.randint(-8, 9, (n, 1), generator=gen, device=DEV).float()


@pytest.mark.parametrize("n,vocab", [(1 << 20, 1000), ((1 << 20) + 1, 300000), (1100000, 60000), (3000000, 1000),
                                     ((1 << 22) + 77, 300000), (5000000, 3000000)])
def test_sums_are_exact(n, vocab):
    tokens, rows = case(n, vocab)
    t, x = tokens.cpu().numpy(), rows.cpu().numpy()[:, 0]
    live = (t >= 0) & (t < vocab)
    want = np.bincount(t[live], weights=x[live], minlength=vocab)
    got = M.embed_grad(tokens, rows, vocab)
    assert np.array_equal(got.cpu().numpy()[:, 0], want)


def test_time_grows_as_the_tokens_do():
    """Four times the tokens may take six times as long, not sixteen."""
    def seconds(n):
        tokens, rows = case(n, 300000)
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        times = []
        for _ in range(4):
            start.record()
            M.embed_grad(tokens, rows, 300000)
            end.record()
            end.synchronize()
            times.append(start.elapsed_time(end))
        return min(times[1:])
    few, many = seconds(1 << 22), seconds(1 << 24)
    print(few, many)
    assert many <= 6 * few
