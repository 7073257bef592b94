"""GPU: the group norm's gradient where a team of threads goes through many batch rows, and where the parts of dweight and
dbias are joined in two and three steps of 512 rows; and inputs whose mean is far from 0.

Tolerances of test_gpu_norm.py, whose bounds for sums go by the sums of sizes: 64 u, u = 2^-24, of which a team's 64
rows one after the other lose 8 at random and a step of the join 16 + 5 at worst.  The reference here is one of whole
arrays, with lengths as masks."""
import pytest
import torch

import paper_1805_11144_amd as M
from test_gpu_norm import BF16, F32, check, inputs

pytestmark = pytest.mark.gpu

# batch, positions, groups, channels of a group
TEAMS = [(2500, 1, 16, 128), (1701, 1, 16, 128), (1100, 1, 2, 1032), (1300, 1, 2, 700), (9001, 1, 40, 24), (300001, 1, 1, 4),
         (70000, 1, 3, 5), (1025, 1, 1, 4100), (700, 1, 9000, 4), (300, 1, 110, 1100)]
RUNS = [(2048, 3, 4, 8), (700, 3, 2, 5), (513, 40, 2, 3), (1025, 2, 1, 1), (270000, 2, 1, 2), (262145, 3, 2, 1)]


def reference(i, g, act, eps=1e-5):
    x, dy = (i[n].double().cpu() for n in ("x", "dy"))
    b, t, c = x.shape
    x, dy = x.view(b, t, g, -1), dy.view(b, t, g, -1)
    w, a = (i[n].double().cpu().view(g, -1) for n in ("weight", "bias"))
    n = torch.full((b,), t) if i["lengths"] is None else i["lengths"].cpu().clamp(0, t).long()
    inside = (torch.arange(t) < n[:, None])[:, :, None, None]
    x, dy = torch.where(inside, x, 0.0), torch.where(inside, dy, 0.0)
    count = (n.clamp(min=1) * (c // g)).double()[:, None, None, None]
    mean = x.sum((1, 3), keepdim=True) / count
    x = torch.where(inside, x - mean, 0.0)
    rstd = (x.square().sum((1, 3), keepdim=True) / count + eps).rsqrt()
    h = x * rstd
    z = h * w + a
    s = torch.sigmoid(z)
    y = torch.where(inside, z * s if act == "silu" else z, 0.0)
    by = torch.where(inside, 1e-5 * (1 + z.abs()) * (1 + 0.05 * (mean * rstd).abs()), 0.0)
    d = dy * (s * (1 + z * (1 - s))) if act == "silu" else dy
    dw, db = (d * h).sum((0, 1)), d.sum((0, 1))
    bw, bb = ((d * h).abs() + (dy * h).abs()).sum((0, 1)), 1.1 * dy.abs().sum((0, 1))
    d = d * w
    dx = rstd * (d - d.sum((1, 3), keepdim=True) / count - h * ((d * h).sum((1, 3), keepdim=True) / count))
    # h, good to 30 u |mean| rstd, is a factor in two of dx's terms; where a group is two or three values that nearly
    # coincide, rstd is up to 316 and this is most of the error
    bx = rstd * (2e-5 + 60 * 2.0 ** -24 * (mean * rstd).abs()) * ((dy * w).abs() * (1 + h.abs())).amax((1, 3), keepdim=True)
    tol = 64 * 2.0 ** -24
    return dict(y=(y.view(b, t, c), by.view(b, t, c)), dx=(torch.where(inside, dx, 0.0).view(b, t, c), (bx * inside).expand(
        b, t, g, c // g).reshape(b, t, c)), dweight=(dw.view(-1), tol * bw.view(-1)), dbias=(db.view(-1), tol * bb.view(-1)))


def compared(i, g, act):
    args = dict(weight=i["weight"], bias=i["bias"], activation=act, lengths=i["lengths"])
    y, kept = M.group_norm(i["x"], g, keep=True, **args)
    grads = M.group_norm_grad(i["x"], g, kept, i["dy"], **args)
    want = reference(i, g, act)
    for name, x in zip(("y", "dx", "dweight", "dbias"), (y, *grads)):
        check(x, want[name], f"{name} {act}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("shape", TEAMS + RUNS)
def test_many_rows(shape, ragged, dtype):
    compared(inputs(*shape, dtype, 51, ragged), shape[2], "silu" if ragged else "none")


# ------------------------------------------------------------------------ far means
# All channels of a group about one number, far larger than the deviation.  A mean in 32 bits is a sum of values of one
# sign: at most k additions one after the other and a tree of 8, k = 32 of a thread's values; with the division and its
# own rounding 42 u |mean|.  So h is off by 42 u |mean| rstd, y by that times the weight (1 here), and dx, which is
# rstd (d - mean(d) - h mean(d h)), by rstd times twice that times the largest |d| (1 + |h|).
@pytest.mark.parametrize("mean", [1e3, 1e4])
@pytest.mark.parametrize("shape", [(40, 1, 3, 64), (6, 16, 2, 8), (9, 1, 2, 700), (3, 500, 2, 24), (2, 4000, 1, 96)])
def test_a_mean_far_from_0(shape, mean):
    b, t, g, width = shape
    gen = torch.Generator().manual_seed(b)
    x = torch.randn(shape, generator=gen) + mean * torch.randn(b, 1, g, 1, generator=gen).sign()
    dy = torch.randn(shape, generator=gen)
    xd, d = x.double(), dy.double()
    var, mu = torch.var_mean(xd, (1, 3), correction=0, keepdim=True)
    rstd = var.rsqrt()
    far = (mu * rstd).abs()
    assert float(far.min()) > 500
    h = (xd - mu) * rstd
    off = 42 * 2.0 ** -24 * far
    bounds = 1e-5 * (1 + h.abs()) + off, rstd * (2e-5 + 2 * off) * (d.abs() * (1 + h.abs())).amax((1, 3), keepdim=True)
    dx = rstd * (d - d.mean((1, 3), keepdim=True) - h * (d * h).mean((1, 3), keepdim=True))
    # the variance as the mean square less the mean's square, in 32 bits: what these inputs are there to catch
    naive = (x.square().mean((1, 3), keepdim=True) - x.mean((1, 3), keepdim=True).square()).clamp(min=1e-6)
    assert bool((((x - x.mean((1, 3), keepdim=True)) * naive.rsqrt() - h).abs() > bounds[0]).any())
    x, dy = (v.reshape(b, t, g * width).cuda() for v in (x, dy))
    y, kept = M.group_norm(x, g, eps=0.0, keep=True)
    got, _, _ = M.group_norm_grad(x, g, kept, dy)
    for v, want, bound in ((y, h, bounds[0]), (got, dx, bounds[1])):
        err = (v.double().cpu().view(shape) - want).abs()
        assert (err <= bound).all(), float((err / bound).max())
