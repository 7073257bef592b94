"""GPU: the gated lowpass, its gradient and its single step against 64 bits, step by step.

Tolerances, in units u = 2^-24: a gate is good to k = 8 + 2 |g| units (the exponential's argument loses |g| / ln 2
half units, the rest is a few roundings).  The bound E of a state's error therefore goes through the same filter
as the state, E[t] = a (E[t-1] + k u S[t-1]) + k u (1 - a) |v|, with S the filter of the sizes; joining runs of
steps only puts the same products in another order.  The gradient's goes the same way back.  A result in 16 bits
adds half a unit of its own."""
import math

import numpy as np
import pytest
import torch

import paper_1805_11144_amd as M

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def inputs(b, t, d, dtype, seed, packed=False, ragged=False):
    r = np.random.default_rng([seed, b, t, d])
    v = r.standard_normal((b, t, d))
    g = 2 + 2 * r.standard_normal((b, t, d))
    if packed:
        g[r.random((b, t)) < 0.05] = -np.inf
        g[r.random((b, t)) < 0.02] = np.inf
        g[r.random((b, t)) < 0.02] = -np.finfo(np.float32).max
    put = lambda x, ty: torch.from_numpy(x).to(ty).to(DEV)  # noqa: E731
    lengths = None
    if ragged:
        n = r.integers(0, t + 1, b)
        n[0] = 0
        n[-1] = t
        lengths = put(n, torch.int32)
    return (put(v, dtype), put(g, dtype), put(r.standard_normal((b, d)), F32), lengths,
            put(r.standard_normal((b, t, d)), dtype), put(r.standard_normal((b, d)), F32))


def host(x):
    return x.double().cpu().numpy()


def reference(v, g, y0, lengths, dy, dlast):
    """Results and error bounds of both passes: {name: (value, bound)}."""
    v, g, dy = host(v), host(g), host(dy)
    b, t, d = v.shape
    n = np.full(b, t) if lengths is None else np.clip(lengths.cpu().numpy(), 0, t)
    with np.errstate(over="ignore"):
        a, r = 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))
    k = (8 + 2 * np.minimum(np.abs(g), 100)) * U
    h = host(y0) if y0 is not None else np.zeros((b, d))
    s, e = np.abs(h), np.zeros((b, d))
    y, ye, before, be = np.zeros_like(v), np.zeros_like(v), np.zeros_like(v), np.zeros_like(v)
    for i in range(t):
        live = (i < n)[:, None]
        before[:, i], be[:, i] = h, e
        e = np.where(live, a[:, i] * (e + k[:, i] * s) + k[:, i] * r[:, i] * np.abs(v[:, i]), e)
        s = np.where(live, a[:, i] * s + r[:, i] * np.abs(v[:, i]), s)
        h = np.where(live, a[:, i] * h + r[:, i] * v[:, i], h)
        y[:, i], ye[:, i] = np.where(live, h, 0), np.where(live, e, 0)
    out = {"y": (y, ye), "last": (h, e)}
    m = host(dlast) if dlast is not None else np.zeros((b, d))
    s, e = np.abs(m), np.zeros((b, d))
    dv, dve, dg, dge = (np.zeros_like(v) for _ in range(4))
    for i in range(t - 1, -1, -1):
        live = (i < n)[:, None]
        at, ae, asz = m + dy[:, i], e + U * (s + np.abs(dy[:, i])), s + np.abs(dy[:, i])
        x, kk = before[:, i] - v[:, i], k[:, i]
        dv[:, i] = np.where(live, r[:, i] * at, 0)
        dve[:, i] = np.where(live, r[:, i] * (ae + kk * asz), 0)
        dg[:, i] = np.where(live, a[:, i] * r[:, i] * x * at, 0)
        xe = be[:, i] + U * (np.abs(before[:, i]) + np.abs(v[:, i]))
        dge[:, i] = np.where(live, a[:, i] * r[:, i] * (xe * asz + (np.abs(x) + xe) * (ae + 2 * kk * asz)), 0)
        m = np.where(live, a[:, i] * at, m)
        e = np.where(live, a[:, i] * (ae + kk * asz), e)
        s = np.where(live, a[:, i] * asz, s)
    out.update(dv=(dv, dve), dg=(dg, dge), dy0=(m, e))
    return out


def check(got, want, name):
    value, bound = want
    half = U if got.dtype == F32 else 2.0 ** -8   # bf16 has 8 significant bits
    err = np.abs(host(got) - value)
    bound = bound * (1 + 2 * half) + half * np.abs(value) * 1.01 + 1e-37
    assert np.isfinite(host(got)).all(), name
    assert (err <= bound).all(), (name, float((err / bound).max()))


def both_passes(v, g, y0, lengths, dy, dlast):
    y, last, kept = M.gated_lowpass(v, g, y0=y0, lengths=lengths, keep=True)
    y2, last2 = M.gated_lowpass(v, g, y0=y0, lengths=lengths)
    assert torch.equal(y, y2) and torch.equal(last, last2)
    dv, dg, dy0 = M.gated_lowpass_grad(v, g, kept, dy, dlast=dlast, lengths=lengths)
    return dict(y=y, last=last, dv=dv, dg=dg, dy0=dy0)


SHAPES = [(1, 1, 1), (2, 3, 5), (1, 15, 64), (3, 16, 33), (2, 17, 130), (1, 63, 7), (4, 64, 16), (2, 65, 96),
          (1, 200, 192), (13, 77, 333), (1, 1000, 24), (2, 1025, 12), (300, 20, 3), (1, 4100, 2)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t,d", SHAPES)
def test_both_passes(b, t, d, dtype):
    for packed, ragged in ((False, False), (True, True)):
        v, g, y0, lengths, dy, dlast = inputs(b, t, d, dtype, 1, packed, ragged)
        want = reference(v, g, y0, lengths, dy, dlast)
        for name, x in both_passes(v, g, y0, lengths, dy, dlast).items():
            check(x, want[name], f"{name} packed={packed}")


def test_no_initial_state_no_last_gradient():
    v, g, _, _, dy, _ = inputs(3, 90, 40, F32, 2)
    want = reference(v, g, None, None, dy, None)
    for name, x in both_passes(v, g, None, None, dy, None).items():
        check(x, want[name], name)


def test_lengths_are_clamped():
    v, g, y0, _, dy, dlast = inputs(4, 50, 16, F32, 3)
    lengths = torch.tensor([-5, 0, 50, 1000], dtype=torch.int32, device=DEV)
    want = reference(v, g, y0, lengths, dy, dlast)
    for name, x in both_passes(v, g, y0, lengths, dy, dlast).items():
        check(x, want[name], name)
    _, last = M.gated_lowpass(v, g, y0=y0, lengths=lengths)
    assert torch.equal(last[:2], y0[:2])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_lies_past_a_length_is_not_used(dtype):
    v, g, y0, lengths, dy, dlast = inputs(5, 150, 48, dtype, 4, False, True)
    clean = both_passes(v, g, y0, lengths, dy, dlast)
    past = (torch.arange(150, device=DEV) >= lengths[:, None])[:, :, None]
    for bad in (float("nan"), float("inf"), -float("inf")):
        w = [torch.where(past, bad, x.float()).to(dtype) for x in (v, g, dy)]
        for name, x in both_passes(w[0], w[1], y0, lengths, w[2], dlast).items():
            assert torch.equal(x, clean[name]), name


def test_a_closed_gate_forgets_and_an_open_one_keeps():
    v, g, y0, _, dy, dlast = inputs(2, 300, 20, F32, 5)
    y, last = M.gated_lowpass(v, torch.full_like(g, -math.inf), y0=y0)
    assert torch.equal(y, v) and torch.equal(last, v[:, -1])
    y, last, kept = M.gated_lowpass(v, torch.full_like(g, math.inf), y0=y0, keep=True)
    assert torch.equal(y, y0[:, None].expand_as(y)) and torch.equal(last, y0)
    dv, dg, dy0 = M.gated_lowpass_grad(v, torch.full_like(g, math.inf), kept, dy, dlast=dlast)
    assert (dv == 0).all() and (dg == 0).all()


def test_nan_stays_in_its_channel_and_sequence():
    v, g, y0, _, dy, dlast = inputs(2, 400, 16, F32, 6)
    v[1, 100, 3] = math.nan
    y, last = M.gated_lowpass(v, g, y0=y0)
    bad = torch.isnan(y)
    assert bad[1, 100:, 3].all() and bad.sum() == 300 and torch.isnan(last).sum() == 1


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(dtype):
    """Steps first, channels inside wider rows at any element, broadcast inputs."""
    b, t, d = 3, 90, 24
    v, g, y0, lengths, dy, dlast = inputs(b, t, d, dtype, 7)
    plain = both_passes(v, g, y0, None, dy, dlast)
    first = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (v, g, dy)]
    wide = []
    for k, x in enumerate((v, g, dy)):
        w = torch.full((b, t, d + 7), math.nan, dtype=dtype, device=DEV)
        w[:, :, k + 1:k + 1 + d] = x
        wide.append(w[:, :, k + 1:k + 1 + d])
    apart = [x.permute(2, 0, 1).contiguous().permute(1, 2, 0) for x in (v, g, dy)]
    for a, q, z in (first, wide, apart):
        for name, x in both_passes(a, q, y0, None, z, dlast).items():
            value, ref = host(x), host(plain[name])
            assert np.allclose(value, ref, rtol=2.0 ** -8 if dtype == BF16 else 1e-5, atol=1e-5), name
    for shape in ((1, t, d), (b, 1, d), (1, 1, d)):
        vb = v[:shape[0], :shape[1]].expand(b, t, d)
        want = reference(vb, g, y0, None, dy, dlast)
        for name, x in both_passes(vb, g, y0, None, dy, dlast).items():
            check(x, want[name], name)


def test_gradient_against_differences():
    """Of sum(w y) + sum(u last) in 64 bits, along random directions of every input."""
    b, t, d = 2, 40, 6
    v, g, y0, _, w, u = inputs(b, t, d, F32, 8)
    _, _, kept = M.gated_lowpass(v, g, y0=y0, keep=True)
    grads = M.gated_lowpass_grad(v, g, kept, w, dlast=u)

    def value(v, g, y0):
        h, total = y0, 0.0
        for i in range(t):
            a = 1 / (1 + np.exp(-g[:, i]))
            h = a * h + (1 - a) * v[:, i]
            total += (host(w)[:, i] * h).sum()
        return total + (host(u) * h).sum()

    r = np.random.default_rng(9)
    at = [host(x) for x in (v, g, y0)]
    for k, grad in enumerate(grads):
        z = r.standard_normal(at[k].shape)
        up, down = list(at), list(at)
        up[k], down[k] = at[k] + 1e-5 * z, at[k] - 1e-5 * z
        slope = (value(*up) - value(*down)) / 2e-5
        size = np.abs(host(grad) * z).sum()
        assert abs(slope - (host(grad) * z).sum()) <= 1e-5 * size + 1e-6


def test_no_steps_no_rows():
    y0 = torch.randn(3, 8, device=DEV)
    empty = torch.empty(3, 0, 8, device=DEV)
    y, last, kept = M.gated_lowpass(empty, empty, y0=y0, keep=True)
    assert y.shape == (3, 0, 8) and torch.equal(last, y0)
    assert (M.gated_lowpass(empty, empty)[1] == 0).all()
    dv, dg, dy0 = M.gated_lowpass_grad(empty, empty, kept, empty, dlast=y0)
    assert torch.equal(dy0, y0)
    none = torch.empty(0, 5, 8, device=DEV)
    assert M.gated_lowpass(none, none)[0].shape == (0, 5, 8)


def test_offsets_past_32_bits():
    """More than 2^31 values in one row: a gate that forgets hands the input through."""
    t, d = 140000, 16384
    v = torch.zeros(1, t, d, dtype=BF16, device=DEV)
    v[0, :, 0] = (torch.arange(t, device=DEV) % 251).to(BF16)
    v[0, -1] = 3.0
    g = torch.full((1, 1, d), -math.inf, dtype=BF16, device=DEV).expand(1, t, d)
    y, last, kept = M.gated_lowpass(v, g.transpose(0, 1).expand(t, 1, d).transpose(0, 1), keep=True)
    assert torch.equal(y[0, :, 0], v[0, :, 0]) and torch.equal(y[0, -70:], v[0, -70:]) and (last == 3).all()
    del y
    dv, dg, dy0 = M.gated_lowpass_grad(v, g, kept, v)
    assert torch.equal(dv[0, :, 0], v[0, :, 0]) and torch.equal(dv[0, -70:], v[0, -70:]) and (dg[0, -70:] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,slots,d", [(1, 1, 1), (3, 9, 17), (8, 64, 1024), (130, 200, 33), (5, 5, 1500)])
def test_step(rows, slots, d, dtype):
    """Single steps, one after another, are the filter's; other slots keep their bits."""
    t = 6
    v, g, y0, _, dy, dlast = inputs(rows, t, d, dtype, 10)
    want = reference(v, g, y0, None, dy, dlast)
    r = np.random.default_rng([11, rows])
    at = torch.from_numpy(r.permutation(slots)[:rows].astype(np.int32)).to(DEV)
    state = torch.randn(slots, d + 3, device=DEV)[:, 2:2 + d]
    state[at.long()] = y0
    before = state.clone()
    for i in range(t):
        y = M.gated_lowpass_step(v[:, i], g[:, i], state, slots=at)
        check(y, (want["y"][0][:, i], want["y"][1][:, i]), f"y {i}")
    check(state[at.long()], want["last"], "state")
    rest = torch.ones(slots, dtype=torch.bool, device=DEV)
    rest[at.long()] = False
    assert torch.equal(state[rest], before[rest])


def test_step_without_slots_and_idle_rows():
    v, g, y0, _, _, _ = inputs(6, 1, 40, F32, 12)
    v, g = v[:, 0], g[:, 0]
    a, b = y0.clone(), y0.clone()
    ya = M.gated_lowpass_step(v, g, a)
    yb = M.gated_lowpass_step(v, g, b, slots=torch.arange(6, dtype=torch.int32, device=DEV))
    assert torch.equal(a, b) and torch.equal(ya, yb) and torch.equal(ya, a)
    c = y0.clone()
    slots = torch.tensor([-1, 6, 2, -2 ** 31, 2 ** 31 - 1, 4], dtype=torch.int32, device=DEV)
    v[0] = math.nan
    yc = M.gated_lowpass_step(v, g, c, slots=slots)
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < 6:
            assert torch.equal(yc[i], c[s])
        else:
            assert (yc[i] == 0).all()
    for s in (0, 1, 3, 5):
        assert torch.equal(c[s], y0[s])


def test_another_stream_and_a_graph():
    v, g, y0, lengths, dy, dlast = inputs(3, 500, 64, F32, 13, False, True)
    want = both_passes(v, g, y0, lengths, dy, dlast)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        w = [x.clone() for x in (v, g, y0, lengths, dy, dlast)]
        got = both_passes(*w)
    side.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)
    state = y0.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, last, kept = M.gated_lowpass(v, g, y0=y0, lengths=lengths, keep=True)
        dv, dg, dy0 = M.gated_lowpass_grad(v, g, kept, dy, dlast=dlast, lengths=lengths)
        M.gated_lowpass_step(v[:, 0], g[:, 0], state)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        sign = 1.0 if k % 2 == 0 else -1.0
        for name, x in dict(y=y, last=last, dv=dv, dg=dg, dy0=dy0).items():
            # the values and what flows back both change sign: dg, their product, does not
            assert torch.equal(x, want[name] * (1.0 if name == "dg" else sign)), name
        for x in (v, y0, dy, dlast):
            x.mul_(-1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,t,d", [(2, 3000, 130), (1, 2113, 257), (70, 600, 31), (40, 1700, 1024)])
def test_many_chunks(b, t, d, dtype):
    """Chunks side by side over several spans, and one after the other in many workgroups."""
    v, g, y0, lengths, dy, dlast = inputs(b, t, d, dtype, 14, True, True)
    want = reference(v, g, y0, lengths, dy, dlast)
    got = both_passes(v, g, y0, lengths, dy, dlast)
    for name, x in got.items():
        check(x, want[name], name)
    again = both_passes(v, g, y0, lengths, dy, dlast)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_any_nan_travels_between_chunks(dtype):
    """NaN of every bit pattern in the inputs, all ones among them."""
    b, t, d = 1, 3000, 8
    v, g, y0, _, dy, dlast = inputs(b, t, d, dtype, 15)
    raw = torch.int32 if dtype == F32 else torch.int16
    v.view(raw)[0, 200, 1] = -1
    g.view(raw)[0, 200, 2] = -1
    y0.view(torch.int32)[0, 3] = -1
    dy.view(raw)[0, 2500, 4] = -1
    dlast.view(torch.int32)[0, 5] = -1
    y, last, kept = M.gated_lowpass(v, g, y0=y0, keep=True)
    bad = torch.isnan(y[0])
    assert bad[200:, 1].all() and bad[200:, 2].all() and bad[:, 3].all() and not bad[:200, 1:3].any()
    assert not bad[:, [0, 4, 5, 6, 7]].any() and torch.isnan(last[0]).tolist() == [False] + [True] * 3 + [False] * 4
    dv, dg, dy0 = M.gated_lowpass_grad(v, g, kept, dy, dlast=dlast)
    assert torch.isnan(dv[0, :2501, 4]).all() and not torch.isnan(dv[0, 2501:, 4]).any() and torch.isnan(dv[0, :, 5]).all()
    assert torch.isnan(dy0[0, 2]) and torch.isnan(dy0[0, 4]) and torch.isnan(dy0[0, 5]) and not torch.isnan(dy0[0, 6])


def test_outputs_in_wider_arrays_through_the_c_call():
    """y with strides of its own: steps first, inside wider rows; nothing around it is written."""
    import ctypes as C

    from paper_1805_11144_amd import mergesim as MS
    b, t, d = 3, 700, 40
    v, g, y0, lengths, _, _ = inputs(b, t, d, F32, 16, True, True)
    want, last = M.gated_lowpass(v, g, y0=y0, lengths=lengths)
    wide = torch.full((t, b, d + 8), 7.0, device=DEV)
    desc = MS.GatedLowpassDesc(batch=b, steps=t, dim=d, dtype=MS.DTYPE_F32, device=0,
                               stream=torch.cuda.current_stream().cuda_stream)
    desc.y_stride[0], desc.y_stride[1] = d + 8, b * (d + 8)
    n = C.c_int64()
    assert MS.load_library().ms_gated_lowpass_workspace(desc, C.byref(n)) == 0
    ws = torch.empty(max(n.value, 1), dtype=torch.uint8, device=DEV)
    got = torch.empty_like(last)
    code = MS.load_library().ms_gated_lowpass(desc, v.data_ptr(), g.data_ptr(), y0.data_ptr(), lengths.data_ptr(),
                                              wide[:, :, 4:].data_ptr(), got.data_ptr(), None, ws.data_ptr(), n.value)
    assert code == 0
    assert torch.equal(wide[:, :, 4:4 + d].transpose(0, 1), want) and torch.equal(got, last)
    assert (wide[:, :, :4] == 7).all() and (wide[:, :, 4 + d:] == 7).all()
