"""GPU: the operators under torch's automatic differentiation, which they take no part in: an argument that asks for
a gradient is refused, and arrays that are written in place say so, so that a backward pass which saved them raises."""
import pytest
import torch

import paper_1805_11144_amd as M

pytestmark = pytest.mark.gpu
DEV = "cuda"


def calls():
    """Each call on fresh arguments: (call, its floating-point arguments by name, the written ones)."""
    def r(*shape):
        return torch.randn(*shape, device=DEV)
    tokens = torch.tensor([1, 0, 3], device=DEV)
    v, g = r(2, 20, 8), r(2, 20, 8)
    kept = M.gated_lowpass(v, g, keep=True)[2]
    return [
        (lambda a: M.embed(tokens, a["table"]), dict(table=r(4, 8)), ()),
        (lambda a: M.embed(tokens, a["table"], out=a["out"]), dict(table=r(4, 8), out=r(3, 8)), ("out",)),
        (lambda a: M.embed_grad(tokens, a["drows"], 4), dict(drows=r(3, 8)), ()),
        (lambda a: M.embed_grad(tokens, a["drows"], out=a["out"], accumulate=True), dict(drows=r(3, 8), out=r(4, 8)),
         ("out",)),
        (lambda a: M.gated_lowpass(a["v"], a["g"], y0=a["y0"], keep=True), dict(v=r(2, 20, 8), g=r(2, 20, 8), y0=r(2, 8)),
         ()),
        (lambda a: M.gated_lowpass_grad(a["v"], a["g"], a["kept"], a["dy"], dlast=a["dlast"]),
         dict(v=v, g=g, kept=kept, dy=r(2, 20, 8), dlast=r(2, 8)), ()),
        (lambda a: M.gated_lowpass_step(a["v"], a["g"], a["state"]), dict(v=r(2, 8), g=r(2, 8), state=r(2, 8)), ("state",)),
        (lambda a: M.gated_lowpass_step(a["v"], a["g"], a["state"], out=a["out"]),
         dict(v=r(2, 8), g=r(2, 8), state=r(2, 8), out=r(2, 8)), ("state", "out")),
        (lambda a: M.orthogonalise(a["x"]), dict(x=r(9, 7)), ()),
        (lambda a: M.orthogonalise(a["x"], out=a["out"]), dict(x=r(9, 7), out=r(9, 7)), ("out",)),
        (lambda a: M.orthogonal_update(a["weight"], a["momentum"], a["grad"], rate=0.1),
         dict(weight=r(9, 7), momentum=r(9, 7), grad=r(9, 7)), ("weight", "momentum")),
    ]


@pytest.mark.parametrize("k", range(11))
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
        a[name].requires_grad_(False)
        call(a)


@pytest.mark.parametrize("k", range(11))
def test_written_arrays_say_so(k):
    call, args, written = calls()[k]
    before = {n: x._version for n, x in args.items()}
    call(args)
    for n, x in args.items():
        assert (x._version > before[n]) == (n in written), n


def test_a_backward_pass_that_saved_a_written_array_raises():
    w, x = torch.randn(9, 7, device=DEV), torch.randn(7, 3, device=DEV, requires_grad=True)
    loss = torch.matmul(w, x).sum()
    M.orthogonal_update(w, torch.zeros_like(w), torch.randn(9, 7, device=DEV), rate=0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_inference_mode():
    with torch.inference_mode():
        state = torch.zeros(2, 8, device=DEV)
        v = torch.randn(2, 8, device=DEV)
        assert torch.equal(M.gated_lowpass_step(v, torch.zeros_like(v), state), 0.5 * v)
    with pytest.raises(RuntimeError, match="[Ii]nference"):
        M.gated_lowpass_step(v, torch.zeros_like(v), state)
    assert torch.equal(state, 0.5 * v)
