"""The operators under torch's forward mode, which they take no part in either: an array that carries a tangent is refused.
A dual tensor does not require a gradient, and its tangent was lost without a word.  The check looks at no GPU."""
import pytest
import torch
import torch.autograd.forward_ad as forward

import paper_1805_11144_amd.operators as O


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    monkeypatch.setattr(O, "_torch", torch)
    monkeypatch.setattr(O, "_forward", forward)


def test_an_array_with_a_tangent_is_refused():
    x = torch.randn(3, 4)
    O._undifferentiated(x, "x")
    with forward.dual_level():
        O._undifferentiated(x, "x")
        dual = forward.make_dual(x, torch.ones_like(x))
        for t in (dual, dual.view(4, 3), dual * 2):
            with pytest.raises(ValueError, match="x carries a tangent"):
                O._undifferentiated(t, "x")
        with torch.no_grad(), pytest.raises(ValueError, match="tangent"):   # which does not turn forward mode off
            O._undifferentiated(dual, "x")
        O._undifferentiated(forward.unpack_dual(dual).primal, "x")
        with torch.inference_mode():
            O._undifferentiated(dual, "x")
    O._undifferentiated(dual, "x")


def test_inside_a_function_transform():
    def f(x):
        with pytest.raises(ValueError, match="tangent"):
            O._undifferentiated(x, "x")
        return x
    x = torch.randn(3)
    torch.func.jvp(f, (x,), (x,))
