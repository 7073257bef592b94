"""GPU: the gated delta rule, its gradient and its single step against 64 bits, step by step.

Tolerances, in units u = 2^-24.  Keys have length one and rates are in [0, 1], so a step P - b k k'P does not stretch
an error, and what is forgotten shrinks it.  Relative to the sizes that go through the same sums (`size`, the rule on
absolute values would overstate it; here the largest entry of a result's row, head and kind stands for it), a step
adds about 3 roundings of 32-bit sums over up to 128 keys (sqrt(128) u at worst in one direction, 12 u), 4 u of the
parts' product and 2 u + |decay| u of the decays.  Errors of independent steps add as their squares and the state
remembers 1 / (1 - a) < 1000 of them in these inputs: at most 32 * 20 u = 4e-5 of the largest entry; a run of a few
hundred steps stays below half of it.  A gradient passes twice through as many.  A result in 16 bits adds half a unit
of its own.  The decays' gradient is <a (H - k x'), S> of every step, here the inner product <H, S> behind the chunk
and differences of it from step to step: its errors go by the sums of |H| |S|, the largest of a row and head, and not
by what is left after products of both signs have cancelled (all of it where a is 0)."""
import numpy as np
import pytest
import torch

import paper_1805_11144_amd as M

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
TOL = {"y": 2e-5, "last": 2e-5, "dq": 4e-5, "dk": 4e-5, "dv": 4e-5, "ddecay": 4e-5, "drate": 4e-5, "ds0": 4e-5}


def inputs(b, t, hk, h, dk, dv, dtype, seed, packed=False, ragged=False):
    r = np.random.default_rng([seed, b, t, hk, h, dk, dv])
    put = lambda x, ty: torch.from_numpy(x).to(ty).to(DEV)  # noqa: E731

    def unit(*shape):
        x = r.standard_normal(shape)
        return put(x / np.linalg.norm(x, axis=-1, keepdims=True), dtype)
    decay = -np.log1p(np.exp(-(4 + 2 * r.standard_normal((b, t, h)))))
    rate = 1 / (1 + np.exp(-r.standard_normal((b, t, h))))
    if packed:
        decay[r.random((b, t)) < 0.03] = -np.inf
        decay[r.random((b, t)) < 0.02] = -np.finfo(np.float32).max
        decay[r.random((b, t)) < 0.02] = 0.0
        rate[r.random((b, t)) < 0.05] = 0.0
        rate[r.random((b, t)) < 0.05] = 1.0
    lengths = None
    if ragged:
        n = r.integers(0, t + 1, b)
        n[0] = 0
        n[-1] = t
        lengths = put(n, torch.int32)
    return dict(q=unit(b, t, hk, dk), k=unit(b, t, hk, dk), v=put(r.standard_normal((b, t, h, dv)), dtype),
                decay=put(decay, F32), rate=put(rate, F32), s0=put(0.3 * r.standard_normal((b, h, dk, dv)), F32),
                lengths=lengths, dy=put(r.standard_normal((b, t, h, dv)), dtype),
                dlast=put(0.3 * r.standard_normal((b, h, dk, dv)), F32))


def reference(i, scale=1.0):
    q, k, v, decay, rate, dy = (i[n].double().cpu() for n in ("q", "k", "v", "decay", "rate", "dy"))
    b, t, h, dv = v.shape
    hk, dk = k.shape[2:]
    of = torch.arange(h) // (h // hk)
    q, k = q[:, :, of], k[:, :, of]
    s = i["s0"].double().cpu() if i["s0"] is not None else torch.zeros(b, h, dk, dv, dtype=torch.float64)
    n = torch.full((b,), t) if i["lengths"] is None else i["lengths"].cpu().clamp(0, t)
    a, y, steps = decay.exp(), torch.zeros_like(v), []
    for x in range(t):
        live = (x < n)[:, None, None, None]
        p = a[:, x, :, None, None] * s
        p = torch.where(a[:, x, :, None, None] == 0, 0.0, p)
        z = v[:, x] - (p * k[:, x, :, :, None]).sum(2)
        new = p + k[:, x, :, :, None] * (rate[:, x, :, None] * z)[:, :, None]
        steps.append((p, z, new, live))
        s = torch.where(live, new, s)
        y[:, x] = torch.where(live[..., 0], scale * (s * q[:, x, :, :, None]).sum(2), 0.0)
    out, inner = dict(y=y, last=s), torch.zeros_like(a)
    d = i["dlast"].double().cpu() if i["dlast"] is not None else torch.zeros_like(s)
    g = {m: torch.zeros_like(x) for m, x in (("dq", q), ("dk", k), ("dv", v), ("ddecay", a), ("drate", a))}
    for x in range(t - 1, -1, -1):
        p, z, new, live = steps[x]
        kx, dyx, bx = k[:, x, :, :, None], scale * dy[:, x, :, None], rate[:, x, :, None]
        total = d + q[:, x, :, :, None] * dyx
        inner[:, x] = (total * new).abs().sum((2, 3)) * live[..., 0, 0]
        du = (total * kx).sum(2)
        dp = total - kx * (bx * du)[:, :, None]
        one = dict(dq=(new * dyx).sum(3), dv=bx * du, ddecay=(dp * p).sum((2, 3)), drate=(du * z).sum(2),
                   dk=(total * (bx * z)[:, :, None]).sum(3) - (p * (bx * du)[:, :, None]).sum(3))
        for m, val in one.items():
            g[m][:, x] = torch.where(live.reshape(b, *[1] * (val.dim() - 1)), val, 0.0)
        d = torch.where(live, a[:, x, :, None, None] * dp, d)
    for m in ("dq", "dk"):
        g[m] = g[m].reshape(b, t, hk, h // hk, dk).sum(3)
    return dict(out, **g, ds0=d, sizes=dict(ddecay=inner))


def check(got, want, name, size=None):
    assert got.shape == want.shape and torch.isfinite(got).all(), name
    if not want.numel():
        return
    half = 0.0 if got.dtype == F32 else 2.0 ** -8
    x = got.double().cpu()
    # by row and head: the axes that the errors of one memory stay in
    axes = {4: (1, 3), 3: (1,)}[want.dim()] if name not in ("last", "ds0") else (2, 3)
    size = (want if size is None else size).abs().amax(axes, keepdim=True)
    err, bound = (x - want).abs(), TOL[name] * size + half * (want.abs() + TOL[name] * size) + 1e-30
    assert (err <= bound).all(), (name, float((err / bound).max()))


def both_passes(i, scale=1.0):
    args = [i[n] for n in ("q", "k", "v", "decay", "rate")]
    y, last, kept = M.gated_delta(*args, s0=i["s0"], lengths=i["lengths"], scale=scale, keep=True)
    y2, last2 = M.gated_delta(*args, s0=i["s0"], lengths=i["lengths"], scale=scale)
    assert torch.equal(y, y2) and torch.equal(last, last2)
    grads = M.gated_delta_grad(*args, kept, i["dy"], dlast=i["dlast"], lengths=i["lengths"], scale=scale)
    again = M.gated_delta_grad(*args, kept, i["dy"], dlast=i["dlast"], lengths=i["lengths"], scale=scale)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    return dict(zip(("y", "last", "dq", "dk", "dv", "ddecay", "drate", "ds0"), (y, last, *grads)))


# batch, steps, key heads, heads, keys, values
SHAPES = [(1, 1, 1, 1, 1, 1), (2, 3, 1, 2, 5, 3), (1, 31, 1, 1, 16, 16), (2, 32, 2, 2, 32, 17), (1, 33, 1, 3, 33, 70),
          (3, 63, 2, 2, 64, 16), (1, 64, 1, 1, 65, 40), (2, 65, 2, 4, 128, 64), (1, 130, 3, 3, 127, 100),
          (5, 77, 1, 2, 48, 8), (1, 300, 2, 2, 24, 200), (1, 1, 4, 4, 128, 128), (9, 20, 1, 1, 100, 24)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_both_passes(shape, dtype):
    for packed, ragged in ((False, False), (True, True)):
        i = inputs(*shape, dtype, 1, packed, ragged)
        want = reference(i, 0.7)
        for name, x in both_passes(i, 0.7).items():
            check(x, want[name], name, want["sizes"].get(name))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_initial_state_no_last_gradient(dtype):
    i = dict(inputs(2, 90, 2, 2, 40, 24, dtype, 2), s0=None, dlast=None)
    want = reference(i)
    for name, x in both_passes(i).items():
        check(x, want[name], name, want["sizes"].get(name))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_steps(dtype):
    i = inputs(3, 0, 1, 2, 12, 20, dtype, 3)
    r = both_passes(i)
    assert torch.equal(r["last"], i["s0"]) and torch.equal(r["ds0"], i["dlast"]) and r["y"].shape == (3, 0, 2, 20)


def test_no_rows():
    i = inputs(0, 5, 1, 2, 12, 20, F32, 3)
    assert all(x.shape[0] == 0 for x in both_passes(i).values())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_lies_past_the_lengths_is_not_read(dtype):
    i = inputs(4, 100, 1, 2, 24, 40, dtype, 4, ragged=True)
    i["lengths"] = torch.tensor([0, 1, 70, 99], dtype=torch.int32, device=DEV)
    want = both_passes(i)
    for n in ("q", "k", "v", "decay", "rate", "dy"):
        for row, length in enumerate(i["lengths"].tolist()):
            i[n][row, length:] = float("nan")
    for name, x in both_passes(i).items():
        assert torch.equal(x, want[name]), name


def test_a_first_step_that_forgets_takes_nothing_of_s0():
    i = inputs(2, 70, 1, 2, 24, 40, F32, 5)
    i["decay"][:, 0] = -float("inf")
    i["s0"][0], i["s0"][1] = float("nan"), float("inf")
    want = reference(dict(i, s0=torch.zeros_like(i["s0"])))
    r = both_passes(i)
    for name, x in r.items():
        check(x, want[name], name, want["sizes"].get(name))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(dtype):
    i = inputs(3, 70, 2, 4, 24, 40, dtype, 6)
    want = both_passes(i)
    j = dict(i)
    for n in ("q", "k", "v", "decay", "rate", "dy"):
        x = i[n]
        wide = torch.full((*x.shape[:2], x.shape[2] + 3, *x.shape[3:]), float("nan"), dtype=x.dtype, device=DEV)
        wide[:, :, 1:-2] = x
        j[n] = wide[:, :, 1:-2]
    for name, x in both_passes(j).items():
        assert torch.equal(x, want[name]), name
    for n in ("q", "k", "v", "decay", "rate", "dy"):   # steps outside, odd bases, columns apart, broadcast rows
        j[n] = i[n].transpose(0, 1).contiguous().transpose(0, 1)
    for name, x in both_passes(j).items():
        assert torch.equal(x, want[name]), name
    for n in ("q", "v", "dy"):
        j[n] = torch.cat([i[n][..., :1], i[n]], -1)[..., 1:]
    j["k"] = i["k"].transpose(2, 3).contiguous().transpose(2, 3)
    for name, x in both_passes(j).items():
        assert torch.equal(x, want[name]), name
    j = dict(i, dy=i["dy"][:, :1].expand_as(i["dy"]))
    k = dict(i, dy=j["dy"].contiguous())
    for (name, x), y in zip(both_passes(j).items(), both_passes(k).values()):
        assert torch.equal(x, y), name


def test_a_captured_pass_replays():
    i = inputs(2, 150, 1, 2, 64, 64, BF16, 7, ragged=True)
    want = both_passes(i)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both_passes(i)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    args = [i[n] for n in ("q", "k", "v", "decay", "rate")]
    with torch.cuda.graph(g):
        y, last, kept = M.gated_delta(*args, s0=i["s0"], lengths=i["lengths"], keep=True)
        grads = M.gated_delta_grad(*args, kept, i["dy"], dlast=i["dlast"], lengths=i["lengths"])
    for _ in range(3):
        for x in (y, last, *grads):
            x.fill_(7.0)
        g.replay()
        both_passes(i)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, last, *grads), want.values()))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,hk,h,dk,dv", [(1, 1, 1, 1, 1), (3, 1, 2, 5, 3), (8, 4, 4, 64, 64), (2, 1, 3, 128, 130),
                                             (40, 2, 2, 100, 36), (2, 1, 1, 128, 257)])
def test_step(rows, hk, h, dk, dv, dtype):
    i = inputs(rows, 1, hk, h, dk, dv, dtype, 8, packed=rows > 8)
    want = reference(i, 0.7)
    state = torch.randn(rows + 5, h, dk, dv, device=DEV)
    slots = torch.randperm(rows + 5, device=DEV)[:rows].to(torch.int32)
    state[slots.long()] = i["s0"]
    before = state.clone()
    args = [i[n][:, 0] for n in ("q", "k", "v", "decay", "rate")]
    y = M.gated_delta_step(*args, state, slots=slots, scale=0.7)
    check(y[:, None], want["y"], "y")
    check(state[slots.long()], want["last"], "last")
    idle = [s for s in range(rows + 5) if s not in slots.tolist()]
    assert torch.equal(state[idle], before[idle])
    # own slots, slots outside the cache, a strided cache, a result of the caller's
    wide = torch.full((rows, 2, h, dk, dv), 5.0, device=DEV)
    wide[:, 0] = i["s0"]
    slots = torch.arange(rows, dtype=torch.int32, device=DEV)
    slots[0] = -1 if rows % 2 else rows
    out = torch.full((rows, h, dv + 1), 7.0, dtype=dtype, device=DEV)
    assert M.gated_delta_step(*args, wide[:, 0], slots=slots, scale=0.7, out=out[..., :dv]) is not None
    assert (out[0, :, :dv] == 0).all() and (out[..., dv] == 7).all() and (wide[:, 1] == 5).all()
    assert torch.equal(wide[0, 0], i["s0"][0])
    check(out[1:, None, :, :dv], want["y"][1:], "y")
    check(wide[1:, 0], want["last"][1:], "last")


def test_step_that_forgets_takes_nothing_of_its_slot():
    i = inputs(2, 1, 1, 2, 24, 40, F32, 9)
    i["decay"][:] = -float("inf")
    state = torch.full((2, 2, 24, 40), float("nan"), device=DEV)
    y = M.gated_delta_step(*[i[n][:, 0] for n in ("q", "k", "v", "decay", "rate")], state)
    want = reference(dict(i, s0=torch.zeros_like(state)))
    check(y[:, None], want["y"], "y")
    check(state, want["last"], "last")


def test_steps_are_the_whole_sequence():
    i = inputs(3, 50, 2, 4, 32, 48, F32, 10)
    y, last = M.gated_delta(*[i[n] for n in ("q", "k", "v", "decay", "rate")], s0=i["s0"])
    state = i["s0"].clone()
    served = torch.stack([M.gated_delta_step(*[i[n][:, t] for n in ("q", "k", "v", "decay", "rate")], state)
                          for t in range(50)], 1)
    check(served, y.double().cpu(), "y")
    check(state, last.double().cpu(), "last")


def test_gradients_against_differences():
    """Along random directions, in the forward call's own 32 bits: differences of 2e-3 are good to about 1e-3."""
    i = inputs(2, 70, 1, 2, 24, 16, F32, 11)
    r = both_passes(i)
    gen = torch.Generator(device=DEV).manual_seed(1)

    def loss(j):
        y, last = M.gated_delta(*[j[n] for n in ("q", "k", "v", "decay", "rate")], s0=j["s0"])
        return float((y.double() * i["dy"].double()).sum() + (last.double() * i["dlast"].double()).sum())
    for n, g in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("decay", "ddecay"), ("rate", "drate"), ("s0", "ds0")):
        z = torch.randn(i[n].shape, generator=gen, device=DEV)
        z = z * (r[g].double().norm() / (r[g].double() * z.double()).sum().abs()).clamp(max=3).float()
        slope = (loss(dict(i, **{n: i[n] + 1e-3 * z})) - loss(dict(i, **{n: i[n] - 1e-3 * z}))) / 2e-3
        assert abs(slope - float((r[g].double() * z.double()).sum())) <= 2e-3 * float(r[g].norm() * 3 + 1), n


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["one key", "long keys", "two keys", "large values", "small values", "short keys", "strong decays"])
def test_inputs_far_from_ordinary_ones(kind, dtype):
    """Keys that repeat without forgetting (a step then undoes the one before it), keys that a step overshoots with,
    values and keys of other sizes: the bounds are relative, and hold as they are."""
    i = inputs(1, 320, 1, 2, 64, 48, dtype, 12)
    if kind == "one key":
        i.update(k=i["k"][:, :1].expand_as(i["k"]), rate=torch.ones_like(i["rate"]), decay=torch.zeros_like(i["decay"]))
    elif kind == "long keys":
        i.update(k=i["k"] * 1.3, rate=torch.ones_like(i["rate"]), decay=torch.zeros_like(i["decay"]))
    elif kind == "two keys":
        i.update(k=i["k"][:, :2].repeat(1, 160, 1, 1), rate=torch.full_like(i["rate"], 0.9))
    elif kind in ("large values", "small values"):
        f = 1e5 if kind == "large values" else 1e-20
        i.update(v=(i["v"].float() * f).to(dtype), s0=i["s0"] * f)
    elif kind == "short keys":
        i.update(k=(i["k"].float() * 1e-3).to(dtype))
    else:
        i.update(decay=i["decay"] * 100)
    want = reference(i)
    for name, x in both_passes(i).items():
        check(x, want[name], name, want["sizes"].get(name))
