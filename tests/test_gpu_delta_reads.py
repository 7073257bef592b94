"""GPU: what the gated delta rule reads is 32 bits wide before it is rounded, also where it is rounded to 16.

Each case reads, at a query of two ones, two numbers of size 1000 to 2000 that nearly cancel, so that the result's own
half unit (2^-8 of it) is far below what 16 bits of the two numbers would lose: a number in [1024, 2048) is held by two
bf16 parts to 2^-7 = 8e-3, by 24 bits to 2^-14 = 6e-5.  In units u = 2^-24 of the sum of sizes that pass through a
result: the parts' products are exact, a sum of them is rounded once for each of up to three products and four runs of
32 keys, of which the largest parts' comes last (3 u and what the small ones add, 1 u); an error z goes through such a
sum three times (P'k, T z, the reads).  12 u covers all; in these inputs it is 2e-3 to 5e-3, and two parts miss it by
up to 2e-2."""
import numpy as np
import pytest
import torch

import paper_1805_11144_amd as M

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def put(x, ty=F32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(ty).to("cuda")


def near(y, want, size):
    want = torch.from_numpy(want)
    half = 2.0 ** -8 if y.dtype == BF16 else 0.0
    bound = 12 * 2.0 ** -24 * size + half * want.abs()
    err = (y.double().cpu() - want).abs()
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("keys", [16, 64, 100, 128])
def test_a_read_of_the_state_that_cancels(keys, dtype):
    r = np.random.default_rng(keys)
    steps, heads, values = 70, 2, 40
    one, two = r.permutation(keys)[:2]
    s0 = r.standard_normal((1, heads, keys, values)).astype(np.float32)
    s0[:, :, one] = r.uniform(1024, 2048, (1, heads, values))
    s0[:, :, two] = -s0[:, :, one] + 0.01 * r.standard_normal((1, heads, values))
    q = np.zeros((1, steps, 1, keys))
    q[..., [one, two]] = 1
    k, v = r.standard_normal((1, steps, 1, keys)) / keys ** 0.5, r.standard_normal((1, steps, heads, values))
    zeros = torch.zeros(1, steps, heads, device="cuda")   # nothing is forgotten, nothing learned
    y, last = M.gated_delta(put(q, dtype), put(k, dtype), put(v, dtype), zeros, zeros, s0=put(s0))
    want = s0[:, :, one].astype(np.float64) + s0[:, :, two]
    near(y, np.repeat(want[:, None], steps, 1), 2 * 2048.0)
    assert torch.equal(last, put(s0))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("keys", [16, 64, 100, 128])
def test_a_read_of_errors_that_cancels(keys, dtype):
    """Two steps put values near 1 in the place of large ones at two keys: what a query of both reads are those, a sum
    of the state before and of two errors of its size."""
    r = np.random.default_rng(keys)
    steps, heads, values = 20, 2, 40
    one, two = r.permutation(keys)[:2]
    s0 = np.zeros((1, heads, keys, values), np.float32)
    s0[:, :, [one, two]] = r.uniform(1024, 2048, (1, heads, 2, values)).astype(np.float32)
    q, k = np.zeros((1, steps, 1, keys)), np.zeros((1, steps, 1, keys))
    q[..., [one, two]] = 1
    k[:, 0, :, one] = k[:, 1, :, two] = 1
    v = r.standard_normal((1, steps, heads, values))
    rate = np.zeros((1, steps, heads))
    rate[:, :2] = 1
    v16 = put(v, dtype)
    y, _ = M.gated_delta(put(q, dtype), put(k, dtype), v16, torch.zeros(1, steps, heads, device="cuda"), put(rate),
                         s0=put(s0))
    want = v16.double().cpu().numpy()[:, :2].sum(1)
    near(y[:, 1:], np.repeat(want[:, None], steps - 1, 1), 4 * 2048.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("keys", [16, 64, 100, 128])
def test_learned_values_that_cancel(keys, dtype):
    """Two steps learn x and -x with nearly equal rates of 24 bits; a query of both keys reads the rates' difference."""
    r = np.random.default_rng(keys)
    steps, heads, values = 20, 3, 40
    one, two = r.permutation(keys)[:2]
    q, k = np.zeros((1, steps, 1, keys)), np.zeros((1, steps, 1, keys))
    q[..., [one, two]] = 1
    k[:, 0, :, one] = k[:, 1, :, two] = 1
    x = put(r.uniform(1024, 2048, (1, heads, values)), BF16).float().cpu().numpy()
    v = np.zeros((1, steps, heads, values))
    v[:, 0], v[:, 1] = x, -x
    rate = np.zeros((1, steps, heads), np.float32)
    rate[:, 0] = r.uniform(0.5, 1, (1, heads))
    rate[:, 1] = rate[:, 0] * (1 + 1e-5 * r.standard_normal((1, heads)))
    y, _ = M.gated_delta(put(q, dtype), put(k, dtype), put(v, dtype), torch.zeros(1, steps, heads, device="cuda"), put(rate))
    d = rate[:, 0].astype(np.float64) - rate[:, 1]
    near(y[:, 1:], np.repeat((d[..., None] * x)[:, None], steps - 1, 1), 2 * 2048.0)
