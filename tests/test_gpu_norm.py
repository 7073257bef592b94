"""GPU: group norm with an activation and its gradient against 64 bits.

Tolerances, in units u = 2^-24.  Inputs have a mean of up to 3 and a deviation near 1.5 (one test: 1000), so h, at most
about 6, is off by 3 u of its terms, u |mean| rstd of the mean and half the variance's relative error; sums of n values
go by trees and runs of at most 64, 12 u at worst.  So h is good to 30 u (1 + |mean| rstd + |h|), z and y to that times
|weight| and |bias|'s 2 u, silu' and silu to 12 u |z| more: 1e-5 of 1 + |y| covers all.  dx is rstd times a difference
of three terms, each good to 60 u of the largest |d weight| (1 + |h|), of which a group's maximum stands for all: 2e-5.
dweight and dbias are sums over rows and positions; their errors are at most 64 u of the sums of sizes (runs of up to
1024 terms one after the other lose sqrt(1024) = 32 u, and 30 of each term).  A 16-bit result adds half a unit."""
import numpy as np
import pytest
import torch

import paper_1805_11144_amd as M

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def inputs(b, t, g, w, dtype, seed, ragged=False, mean=1.0):
    r = np.random.default_rng([seed, b, t, g, w])
    put = lambda x, ty: torch.from_numpy(x).to(ty).to(DEV)  # noqa: E731
    c = g * w
    lengths = None
    if ragged:
        n = r.integers(0, t + 1, b)
        n[0], n[-1] = 0, t
        lengths = put(n, torch.int32)
    return dict(x=put(1.5 * r.standard_normal((b, t, c)) + mean * r.standard_normal(c), dtype),
                weight=put(1 + 0.3 * r.standard_normal(c), F32), bias=put(0.3 * r.standard_normal(c), F32),
                dy=put(r.standard_normal((b, t, c)), dtype), lengths=lengths)


def reference(i, g, act, eps):
    """Results and what their errors go by."""
    x, dy = i["x"].double().cpu(), i["dy"].double().cpu()
    b, t, c = x.shape
    x, dy = x.reshape(b, t, g, c // g), dy.reshape(b, t, g, c // g)
    one = lambda n, v: i[n].double().cpu().reshape(g, -1) if i[n] is not None else torch.full((g, c // g), v).double()  # noqa: E731
    w, a = one("weight", 1.0), one("bias", 0.0)
    y, dx, by, bx = (torch.zeros_like(x) for _ in range(4))
    dw, db, bw, bb = (torch.zeros_like(w) for _ in range(4))
    for row in range(b):
        n = t if i["lengths"] is None else min(max(int(i["lengths"][row]), 0), t)
        if n == 0:
            continue
        v, mean = torch.var_mean(x[row, :n], (0, 2), correction=0, keepdim=True)
        rstd = (v + eps).rsqrt()
        h = (x[row, :n] - mean) * rstd
        z = h * w + a
        s = torch.sigmoid(z)
        y[row, :n] = {"none": z, "relu": z.clamp(min=0), "silu": z * s}[act]
        by[row, :n] = 1e-5 * (1 + z.abs()) * (1 + 0.05 * (mean * rstd).abs())
        d = dy[row, :n] * {"none": torch.ones_like(z), "relu": (z > 0).double(), "silu": s * (1 + z * (1 - s))}[act]
        dw += (d * h).sum(0)
        db += d.sum(0)
        bw += (d * h).abs().sum(0) + (dy[row, :n] * h).abs().sum(0)
        bb += dy[row, :n].abs().sum(0) * 1.1
        d = d * w
        dx[row, :n] = rstd * (d - d.mean((0, 2), keepdim=True) - h * (d * h).mean((0, 2), keepdim=True))
        bx[row, :n] = 2e-5 * rstd * ((dy[row, :n] * w).abs() * (1 + h.abs())).amax((0, 2), keepdim=True)
    tol = 64 * 2.0 ** -24
    return dict(y=(y.reshape(b, t, c), by.reshape(b, t, c)), dx=(dx.reshape(b, t, c), bx.reshape(b, t, c)),
                dweight=(dw.reshape(-1), tol * bw.reshape(-1)), dbias=(db.reshape(-1), tol * bb.reshape(-1)))


def both_passes(i, g, act, eps=1e-5):
    args = dict(weight=i["weight"], bias=i["bias"], activation=act, lengths=i["lengths"])
    y, kept = M.group_norm(i["x"], g, eps=eps, keep=True, **args)
    assert torch.equal(y, M.group_norm(i["x"], g, eps=eps, **args))
    grads = M.group_norm_grad(i["x"], g, kept, i["dy"], **args)
    again = M.group_norm_grad(i["x"], g, kept, i["dy"], **args)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    return dict(zip(("y", "dx", "dweight", "dbias"), (y, *grads)))


def check(got, want, name):
    value, bound = want
    half = 0.0 if got.dtype == F32 else 2.0 ** -8
    x = got.double().cpu()
    assert torch.isfinite(x).all(), name
    bound = bound + half * (value.abs() + bound) + 1e-30
    assert ((x - value).abs() <= bound).all(), (name, float(((x - value).abs() / bound).max()))


# batch, positions, groups, channels of a group
SHAPES = [(1, 1, 1, 1), (3, 1, 2, 5), (70, 1, 16, 128), (9, 1, 3, 37), (5, 1, 2, 700), (3, 1, 1, 5000), (2, 1, 70, 1),
          (4, 7, 3, 6), (2, 16, 4, 16), (3, 100, 2, 10), (1, 1000, 5, 8), (3, 777, 9, 37), (2, 300, 2, 640), (2, 64, 1, 4),
          (300, 3, 1, 8), (1, 40, 1, 2100), (5, 1, 2, 800), (3, 1, 2, 101), (4, 1, 2, 203), (2, 1, 3, 401), (2, 1, 1, 1000),
          (3, 5, 2, 20), (2, 11, 2, 19), (2, 9, 2, 45), (2, 20, 1, 50)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_both_passes(shape, dtype):
    for act, ragged in (("none", False), ("silu", True), ("silu", False)):
        i = inputs(*shape, dtype, 1, ragged)
        want = reference(i, shape[2], act, 1e-5)
        for name, x in both_passes(i, shape[2], act).items():
            check(x, want[name], f"{name} {act} {ragged}")


@pytest.mark.parametrize("shape", [(9, 1, 3, 40), (3, 100, 2, 24)])
def test_relu(shape):
    """No gradient comes in where the corner is within an argument's error."""
    i = inputs(*shape, F32, 2)
    x, w, a = (i[n].double().cpu() for n in ("x", "weight", "bias"))
    v, mean = torch.var_mean(x.reshape(shape[0], shape[1], shape[2], -1), (1, 3), correction=0, keepdim=True)
    z = ((x.reshape(*shape[:3], -1) - mean) * (v + 1e-5).rsqrt()).reshape(x.shape) * w + a
    i["dy"][(z.abs() < 1e-4).to(DEV)] = 0.0
    want = reference(i, shape[2], "relu", 1e-5)
    for name, x in both_passes(i, shape[2], "relu").items():
        check(x, want[name], name)


@pytest.mark.parametrize("shape", [(4, 1, 3, 64), (3, 500, 2, 24)])
def test_without_weight_and_bias_and_a_large_mean(shape):
    i = dict(inputs(*shape, F32, 3, mean=1000.0), weight=None, bias=None)
    want = reference(i, shape[2], "none", 0.0)
    for name, x in both_passes(i, shape[2], "none", 0.0).items():
        value, bound = want[name]   # x itself is known to u |x|: 1000 u in h, and d h cancels nothing of it
        check(x, (value, bound + 1e-3 * 2 ** 0.5 * (1 + value.abs().max()) * 0.2), name)


def test_no_rows_and_no_positions():
    for b, t in ((0, 3), (3, 0), (0, 1)):
        i = inputs(b, t, 2, 8, F32, 4)
        r = both_passes(i, 2, "silu")
        assert r["y"].shape == r["dx"].shape == (b, t, 16)
        assert torch.equal(r["dweight"], torch.zeros(16, device=DEV)) and torch.equal(r["dbias"], torch.zeros(16, device=DEV))


@pytest.mark.parametrize("shape", [(6, 1, 2, 24), (4, 20, 2, 24), (4, 300, 2, 24)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_lies_past_the_lengths_is_not_read(shape, dtype):
    i = inputs(*shape, dtype, 5, ragged=True)
    want = both_passes(i, shape[2], "silu")
    for row, n in enumerate(i["lengths"].tolist()):
        i["x"][row, n:] = float("nan")
        i["dy"][row, n:] = float("inf")
    for name, x in both_passes(i, shape[2], "silu").items():
        assert torch.equal(x, want[name]), name
    i["lengths"] = torch.tensor([-3, 10 ** 6] + [0] * (shape[0] - 2), dtype=torch.int32, device=DEV)   # clamped
    i["x"], i["dy"] = torch.nan_to_num(i["x"]), torch.nan_to_num(i["dy"], posinf=1.0)
    want = reference(i, shape[2], "silu", 1e-5)
    for name, x in both_passes(i, shape[2], "silu").items():
        check(x, want[name], name)


@pytest.mark.parametrize("shape", [(6, 1, 2, 24), (3, 20, 2, 24), (3, 300, 3, 16)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(shape, dtype):
    i = inputs(*shape, dtype, 6)
    want = reference(i, shape[2], "silu", 1e-5)
    whole = both_passes(i, shape[2], "silu")

    def wider(x):
        w = torch.full((x.shape[0], x.shape[1] + 2, x.shape[2] + 8), float("nan"), dtype=x.dtype, device=DEV)
        w[:, 1:-1, 8:] = x
        return w[:, 1:-1, 8:]
    j = dict(i, x=wider(i["x"]), dy=wider(i["dy"]))
    for name, x in both_passes(j, shape[2], "silu").items():
        assert torch.equal(x, whole[name]), name
    # positions outside, odd bases, channels apart, a broadcast gradient
    for change in (lambda x: x.transpose(0, 1).contiguous().transpose(0, 1),
                   lambda x: torch.cat([x[..., :1], x], -1)[..., 1:],
                   lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)):
        j = dict(i, x=change(i["x"]), dy=change(i["dy"]))
        for name, x in both_passes(j, shape[2], "silu").items():
            check(x, want[name], name)
    odd = torch.cat([i["weight"][:1], i["weight"]])[1:]
    for name, x in both_passes(dict(i, weight=odd), shape[2], "silu").items():
        check(x, want[name], name)
    j = dict(i, dy=i["dy"][:, :1, :1].expand_as(i["dy"]))
    k = dict(i, dy=j["dy"].contiguous())
    for (name, x), y in zip(both_passes(j, shape[2], "silu").items(), both_passes(k, shape[2], "silu").values()):
        assert torch.equal(x, y), name


def test_dimensions():
    i = inputs(3, 20, 2, 16, F32, 7)
    want = both_passes(i, 2, "silu")
    j = dict(i, x=i["x"].reshape(3, 4, 5, 32), dy=i["dy"].reshape(3, 4, 5, 32))
    for name, x in both_passes(j, 2, "silu").items():
        assert torch.equal(x.reshape(want[name].shape), want[name]), name
    i = inputs(20, 1, 2, 16, F32, 7)
    want = both_passes(i, 2, "silu")
    for name, x in both_passes(dict(i, x=i["x"][:, 0], dy=i["dy"][:, 0]), 2, "silu").items():
        assert torch.equal(x.reshape(want[name].shape), want[name]), name


@pytest.mark.parametrize("shape", [(40, 1, 4, 64), (3, 400, 2, 24)])
def test_a_captured_pass_replays(shape):
    i = inputs(*shape, BF16, 8, ragged=True)
    want = both_passes(i, shape[2], "silu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both_passes(i, shape[2], "silu")
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    args = dict(weight=i["weight"], bias=i["bias"], activation="silu", lengths=i["lengths"])
    with torch.cuda.graph(g):
        y, kept = M.group_norm(i["x"], shape[2], keep=True, **args)
        out = (y, *M.group_norm_grad(i["x"], shape[2], kept, i["dy"], **args))
    for _ in range(3):
        for x in out:
            x.fill_(7.0)
        g.replay()
        both_passes(i, shape[2], "silu")
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want.values()))


@pytest.mark.parametrize("shape", [(9, 1, 3, 40), (3, 200, 2, 24)])
def test_gradients_against_differences(shape):
    i = inputs(*shape, F32, 9)
    r = both_passes(i, shape[2], "silu")
    gen = torch.Generator(device=DEV).manual_seed(1)

    def loss(j):
        y = M.group_norm(j["x"], shape[2], weight=j["weight"], bias=j["bias"], activation="silu")
        return float((y.double() * i["dy"].double()).sum())
    for n, g in (("x", "dx"), ("weight", "dweight"), ("bias", "dbias")):
        z = torch.randn(i[n].shape, generator=gen, device=DEV)
        slope = (loss(dict(i, **{n: i[n] + 1e-2 * z})) - loss(dict(i, **{n: i[n] - 1e-2 * z}))) / 2e-2
        # third derivatives of size one: 1e-4 of the sizes; 32-bit results: 1e-6 / 1e-2
        assert abs(slope - float((r[g].double() * z.double()).sum())) <= 1e-3 * float((r[g].double() * z.double()).abs().sum() + 1), n
