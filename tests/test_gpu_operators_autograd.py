"""GPU: the operators under torch's automatic differentiation, which they take no part in: an argument that asks for
a gradient is refused."""
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
