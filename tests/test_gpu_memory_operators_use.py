"""GPU: the operators of keyed memories as programs call them: under automatic differentiation, on streams of their own
at the same time, on arrays past 2^31 values, and again on the same arrays."""
import pytest
import torch

import paper_1805_11144_amd as M

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16


def r(*shape):
    return torch.randn(*shape, device=DEV)


def delta_inputs(b=2, t=70, hk=1, h=2, dk=16, dv=24):
    return dict(q=r(b, t, hk, dk) / dk ** 0.5, k=r(b, t, hk, dk) / dk ** 0.5, v=r(b, t, h, dv), decay=-r(b, t, h).abs(),
                rate=torch.sigmoid(r(b, t, h)))


def calls():
    """Each call on fresh arguments: (call, its floating-point arguments by name, the written ones)."""
    d = delta_inputs()
    kept = M.gated_delta(**d, keep=True)[2]
    s = {n: x[:, 0].contiguous() for n, x in delta_inputs().items()}
    x, w = r(5, 12), dict(weight=r(12), bias=r(12))
    stats = M.group_norm(x, 3, **w, keep=True)[1]
    return [
        (lambda a: M.gated_delta(**a, keep=True), dict(d, s0=r(2, 2, 16, 24)), ()),
        (lambda a: M.gated_delta_grad(**a), dict(d, kept=kept, dy=r(2, 70, 2, 24), dlast=r(2, 2, 16, 24)), ()),
        (lambda a: M.gated_delta_step(**a), dict(s, state=r(3, 2, 16, 24)), ("state",)),
        (lambda a: M.gated_delta_step(**a), dict(s, state=r(3, 2, 16, 24), out=r(2, 2, 24)), ("state", "out")),
        (lambda a: M.group_norm(a["x"], 3, weight=a["weight"], bias=a["bias"], activation="silu"), dict(w, x=x), ()),
        (lambda a: M.group_norm_grad(a["x"], 3, a["kept"], a["dy"], weight=a["weight"], bias=a["bias"]),
         dict(w, x=x, kept=stats, dy=r(5, 12)), ()),
    ]


@pytest.mark.parametrize("k", range(6))
def test_arguments_that_ask_for_a_gradient(k):
    call, args, _ = calls()[k]
    for name in args:
        a = {n: x.clone() for n, x in args.items()}
        before = {n: x.clone() for n, x in a.items()}
        a[name].requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            call(a)
        assert all(torch.equal(a[n], before[n]) for n in a)
        with torch.no_grad():
            call(a)


@pytest.mark.parametrize("k", range(6))
def test_written_arrays_say_so(k):
    call, args, written = calls()[k]
    before = {n: x._version for n, x in args.items()}
    call(args)
    for n, x in args.items():
        assert (x._version > before[n]) == (n in written), n


def test_inference_mode():
    s = {n: x[:, 0].contiguous() for n, x in delta_inputs().items()}
    with torch.inference_mode():
        state = torch.zeros(2, 2, 16, 24, device=DEV)
        M.gated_delta_step(**s, state=state)
    with pytest.raises(RuntimeError, match="[Ii]nference"):
        M.gated_delta_step(**s, state=state)


@pytest.mark.parametrize("bad", [
    lambda d: dict(d, q=d["q"][..., :8]), lambda d: dict(d, k=d["k"].half()), lambda d: dict(d, q=d["q"].to(BF16)),
    lambda d: dict(d, decay=d["decay"].to(BF16)), lambda d: dict(d, rate=d["rate"][:, :5]),
    lambda d: dict(d, q=d["q"][0]), lambda d: dict(d, v=d["v"][0]), lambda d: dict(d, s0=r(2, 2, 24, 16)),
    lambda d: dict(d, lengths=torch.zeros(2, dtype=torch.int64, device=DEV)), lambda d: dict(d, decay=d["decay"].cpu()),
    lambda d: dict(d, scale=1e300)])
def test_refusals_of_the_binding(bad):
    with pytest.raises((ValueError, M.MergesimError)):
        M.gated_delta(**bad(delta_inputs()))


def test_refusals_of_the_steps_and_the_norm():
    s = {n: x[:, 0].contiguous() for n, x in delta_inputs().items()}
    for state, out in ((r(2, 2, 24, 16), None), (r(2, 2, 16, 48)[..., :24], None), (r(2, 2, 16, 24).to(BF16), None),
                       (r(2, 2, 16, 24), r(2, 2, 48)[..., ::2]), (r(2, 2, 16, 24), r(2, 24))):
        with pytest.raises(ValueError):
            M.gated_delta_step(**s, state=state, out=out)
    x = r(4, 12)
    for call in (lambda: M.group_norm(x, 5), lambda: M.group_norm(x, 0), lambda: M.group_norm(x, 3, activation="tanh"),
                 lambda: M.group_norm(x, 3, weight=r(11)), lambda: M.group_norm(x, 3, eps=-1.0),
                 lambda: M.group_norm(x[0], 3), lambda: M.group_norm_grad(x, 3, r(4, 3), x),
                 lambda: M.group_norm_grad(x, 3, r(4, 3, 2), x[:3])):
        with pytest.raises((ValueError, M.MergesimError)):
            call()


def test_two_streams_at_once():
    ds = [delta_inputs(4, 300, 2, 4, 64, 64) for _ in range(2)]
    xs = [r(40, 333, 96) for _ in range(2)]

    def all_of(d, x):
        y, last, kept = M.gated_delta(**d, keep=True)
        n, st = M.group_norm(x, 8, activation="silu", keep=True)
        return (y, last, *M.gated_delta_grad(**d, kept=kept, dy=y), n, *M.group_norm_grad(x, 8, st, n, activation="silu"))
    want = [all_of(d, x) for d, x in zip(ds, xs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ds]
    for _ in range(3):
        got = []
        for st, d, x in zip(streams, ds, xs):
            with torch.cuda.stream(st):
                got.append(all_of(d, x))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_two_graphs_share_their_memory():
    """Two captured passes, each with workspaces from torch's pool of one graph, replayed in turn."""
    d, x = delta_inputs(3, 200, 1, 2, 32, 32), r(20, 100, 32)
    want = M.gated_delta(**d), M.group_norm(x, 4, activation="silu")
    torch.cuda.synchronize()
    a, b = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(a):
        y, last = M.gated_delta(**d)
    with torch.cuda.graph(b, pool=a.pool()):
        n = M.group_norm(x, 4, activation="silu")
    for _ in range(3):
        a.replay()
        first = y.clone(), last.clone()
        b.replay()
        torch.cuda.synchronize()
        assert torch.equal(first[0], want[0][0]) and torch.equal(first[1], want[0][1]) and torch.equal(n, want[1])


def test_a_sequence_past_2_31_values():
    """1048640 steps of 16 heads of 128 values: in one run, and in two, which chunks of 64 steps make the same."""
    t, cut = 1048640, 524288 + 64
    gen = torch.Generator(device=DEV).manual_seed(2)

    def rand(*shape):
        return torch.randn(shape, generator=gen, device=DEV, dtype=BF16)
    d = dict(q=rand(1, t, 1, 16) / 4, k=rand(1, t, 1, 16) / 4, v=rand(1, t, 16, 128),
             decay=-0.05 * rand(1, t, 16).float().abs(), rate=torch.sigmoid(rand(1, t, 16).float()))
    assert d["v"].numel() > 1 << 31
    y, last = M.gated_delta(**d)
    one, state = M.gated_delta(**{n: x[:, :cut] for n, x in d.items()})
    assert torch.equal(y[:, :cut], one)
    del one
    two, state = M.gated_delta(**{n: x[:, cut:] for n, x in d.items()}, s0=state)
    assert torch.equal(y[:, cut:], two) and torch.equal(last, state)


@pytest.mark.parametrize("shape", [(2, 1100000, 1024, 32), (1100000, 1, 2048, 16)])
def test_norms_past_2_31_values(shape):
    b, t, c, g = shape
    x = torch.randn(b, t, c, dtype=BF16, device=DEV)
    w = dict(weight=r(c), bias=r(c), activation="silu")
    y, kept = M.group_norm(x, g, **w, keep=True)
    assert x.numel() > 1 << 31
    dx, dweight, dbias = M.group_norm_grad(x, g, kept, x, **w)
    at = slice(b - 1, b) if t > 1 else slice(b - 5, b)
    tail, ends = M.group_norm(x[at].clone(), g, **w, keep=True)
    if t == 1:   # the same teams
        assert torch.equal(y[at], tail) and torch.equal(kept[at], ends)
        assert torch.equal(dx[at], M.group_norm_grad(x[at].clone(), g, ends, x[at].clone(), **w)[0])
    else:        # other runs: sums in another order
        assert float((y[at].float() - tail.float()).abs().max()) <= 0.04   # a unit of bf16 below 8
        assert torch.allclose(kept[at], ends, rtol=1e-5, atol=1e-5)
    assert torch.isfinite(dweight).all() and torch.isfinite(dbias).all()
    h = (x[:1, :1000].double().reshape(-1, g, c // g) - kept[0 if t > 1 else slice(0, 1), :, 0].double()[..., None]) * \
        kept[0 if t > 1 else slice(0, 1), :, 1].double()[..., None]
    assert float((h.reshape(-1, c) ** 2).mean()) < 2
