"""GPU: the C calls of the keyed memory's operators as the binding does not make them: results at strides of the caller's,
results that are not wanted, workspaces of exactly the size named, a stream that is not torch's."""
import ctypes as C

import pytest
import torch

import paper_1805_11144_amd as M
from paper_1805_11144_amd import mergesim as MS
from test_gpu_delta import BF16, F32, inputs

pytestmark = pytest.mark.gpu
GUARD = 4096


def size(call, *args):
    n = C.c_int64()
    assert getattr(MS.load_library(), call)(*args, C.byref(n)) == 0
    return n.value


class Workspace:
    """n bytes between two runs of a known byte."""

    def __init__(self, n):
        self.n = n
        self.all = torch.full((n + 2 * GUARD,), 77, dtype=torch.uint8, device="cuda")

    def args(self):
        return (self.all.data_ptr() + GUARD if self.n else None), self.n

    def intact(self):
        return bool((self.all[:GUARD] == 77).all()) and bool((self.all[GUARD + self.n:] == 77).all())


def at(x):
    return None if x is None else x.data_ptr()


def run(call, desc, *args):
    """On a stream of its own, behind what torch has enqueued."""
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    desc.stream, desc.device = stream.cuda_stream, 0
    code = getattr(MS.load_library(), call)(C.byref(desc), *args)
    assert code == 0, MS.load_library().ms_last_error()
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()


def delta_desc(i, scale=0.7):
    b, t, hk, dk = i["q"].shape
    h, dv = i["v"].shape[2:]
    return MS.GatedDeltaDesc(batch=b, steps=t, heads=h, key_heads=hk, keys=dk, values=dv, scale=scale,
                             dtype=MS.DTYPE_BF16 if i["q"].dtype == BF16 else MS.DTYPE_F32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("order", [(0, 1, 2), (1, 0, 2), (2, 0, 1), (0, 2, 1), (1, 2, 0)])   # of rows, steps and heads in y
@pytest.mark.parametrize("shape,pad", [((3, 150, 1, 2, 24, 40), 8), ((2, 70, 2, 4, 128, 72), 3), ((2, 131, 1, 2, 128, 64), 0),
                                       ((1, 65, 1, 1, 5, 3), 1)])
def test_y_at_strides_of_the_callers(shape, pad, order, dtype):
    i = inputs(*shape, dtype, 61, packed=True, ragged=shape[0] > 1)
    args = [i[n] for n in ("q", "k", "v", "decay", "rate")]
    want, state = M.gated_delta(*args, s0=i["s0"], lengths=i["lengths"], scale=0.7)
    sizes = [i["v"].shape[n] for n in order]
    wide = torch.full((*sizes, i["v"].shape[3] + pad), 7.0, dtype=dtype, device="cuda")
    y = wide[..., pad:].permute(*[order.index(n) for n in range(3)], 3)
    d = delta_desc(i)
    d.y_stride[:] = y.stride()[:3]
    last = torch.full_like(state, 7.0)
    for keep in (None, last):   # the last state is wanted, or not
        w = Workspace(size("ms_gated_delta_workspace", d, 0))
        run("ms_gated_delta", d, *[at(x) for x in args], at(i["s0"]), at(i["lengths"]), at(y), at(keep), None, *w.args())
        assert w.intact() and torch.equal(y, want) and (wide[..., :pad] == 7).all()
    assert torch.equal(last, state)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_without_ds0_and_workspaces_of_the_size_named(dtype):
    for shape in ((3, 150, 1, 2, 24, 40), (2, 70, 2, 4, 128, 72), (40, 200, 2, 4, 33, 17)):
        i = inputs(*shape, dtype, 62, packed=True, ragged=True)
        args = [i[n] for n in ("q", "k", "v", "decay", "rate")]
        _, _, kept = M.gated_delta(*args, s0=i["s0"], lengths=i["lengths"], scale=0.7, keep=True)
        want = M.gated_delta_grad(*args, kept, i["dy"], dlast=i["dlast"], lengths=i["lengths"], scale=0.7)
        d = delta_desc(i)
        mine = Workspace(4 * size("ms_gated_delta_kept", d))   # kept between guards
        w = Workspace(size("ms_gated_delta_workspace", d, 0))
        y = torch.empty_like(i["v"])
        run("ms_gated_delta", d, *[at(x) for x in args], at(i["s0"]), at(i["lengths"]), at(y), None, mine.args()[0], *w.args())
        assert w.intact() and mine.intact()
        outs = [torch.full_like(x, 7.0) for x in want]
        w = Workspace(size("ms_gated_delta_workspace", d, 1))
        run("ms_gated_delta_grad", d, *[at(x) for x in args], mine.args()[0], at(i["lengths"]), at(i["dy"]), at(i["dlast"]),
            *[at(x) for x in outs[:5]], None, *w.args())
        assert w.intact() and mine.intact()
        assert all(torch.equal(a, b) for a, b in zip(outs[:5], want)) and (outs[5] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("shape,pad", [((5, 1, 4, 24), 8), ((300, 1, 3, 1100), 4), ((4, 30, 2, 24), 8), ((3, 700, 3, 7), 1),
                                       ((600, 3, 2, 5), 0)])
def test_norm_at_strides_of_the_callers(shape, pad, turned, dtype):
    b, t, g, width = shape
    c = g * width
    x, dy = torch.randn(b, t, c, device="cuda").to(dtype), torch.randn(b, t, c, device="cuda").to(dtype)
    weight, bias = torch.randn(c, device="cuda"), torch.randn(c, device="cuda")
    lengths = torch.randint(t + 1, (b,), device="cuda").to(torch.int32)
    w = dict(weight=weight, bias=bias, activation="silu", lengths=lengths)
    want, stats = M.group_norm(x, g, keep=True, **w)
    grads = M.group_norm_grad(x, g, stats, dy, **w)

    def placed(v, fill):
        wide = torch.full(((t, b) if turned else (b, t)) + (c + pad,), fill, dtype=dtype, device="cuda")
        inner = wide[..., pad:].transpose(0, 1) if turned else wide[..., pad:]
        if v is not None:
            inner.copy_(v)
        return wide, inner
    d = MS.GroupNormDesc(batch=b, positions=t, channels=c, groups=g, eps=1e-5, activation=2,
                         dtype=MS.DTYPE_BF16 if dtype == BF16 else MS.DTYPE_F32)
    wide, y = placed(None, 7.0)
    _, xs = placed(x, float("nan"))
    _, ds = placed(dy, float("nan"))
    d.x_stride[:], d.y_stride[:] = xs.stride()[:2], y.stride()[:2]
    kept = torch.full((b, g, 2), 7.0, device="cuda")
    # another word makes other sums: a bf16 result is one rounding off at most, a float32 one a few
    near = dict(rtol=2.0 ** -7, atol=1e-5) if dtype == BF16 else dict(rtol=1e-5, atol=1e-5)
    for keep in (None, kept):
        ws = Workspace(size("ms_group_norm_workspace", d, 0))
        run("ms_group_norm", d, at(xs), at(weight), at(bias), at(lengths), at(y), at(keep), *ws.args())
        assert ws.intact() and (wide[..., :pad] == 7).all()
        assert torch.allclose(y.float(), want.float(), **near)
    assert torch.allclose(kept, stats, rtol=1e-5, atol=1e-6)
    ws = Workspace(size("ms_group_norm_workspace", d, 1))
    outs = [torch.full_like(v, 7.0) for v in grads]
    run("ms_group_norm_grad", d, at(xs), at(weight), at(bias), at(lengths), at(kept), at(ds), *[at(v) for v in outs], *ws.args())
    assert ws.intact()
    for got, ref in zip(outs, grads):
        scale = float(ref.float().abs().max()) or 1.0
        assert float((got.float() - ref.float()).abs().max()) <= scale * (2.0 ** -7 if got.dtype == BF16 else 2e-5)
