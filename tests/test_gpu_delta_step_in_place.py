"""GPU: the gated delta rule's step whose result takes the place of v, or lies between other arrays of one buffer, gives
the bits of one with a result of its own."""
import pytest
import torch

import paper_1805_11144_amd as M

pytestmark = pytest.mark.gpu


def arrays(rows, hk, h, dk, dv, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows + dv)

    def r(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    return dict(q=(r(rows, hk, dk) / dk ** 0.5).to(dtype), k=(r(rows, hk, dk) / dk ** 0.5).to(dtype), v=r(rows, h, dv).to(dtype),
                decay=-r(rows, h).abs(), rate=torch.sigmoid(r(rows, h))), r(rows + 3, h, dk, dv)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,hk,h,dk,dv", [(200, 4, 8, 128, 128), (1, 1, 1, 128, 128), (64, 1, 2, 100, 37), (9, 2, 2, 128, 260)])
def test_the_result_in_the_place_of_v(rows, hk, h, dk, dv, dtype):
    a, state = arrays(rows, hk, h, dk, dv, dtype)
    slots = torch.randperm(rows + 3, device="cuda")[:rows].to(torch.int32)
    slots[rows // 2] = -1
    first = state.clone()
    want = M.gated_delta_step(**a, state=first, slots=slots)
    for strided in (False, True):
        v = a["v"].clone()
        if strided:   # behind other columns of a wider buffer
            wide = torch.full((rows, h * dv + 8), 3.0, dtype=dtype, device="cuda")
            v = wide[:, 8:].view(rows, h, dv)
            v.copy_(a["v"])
        second = state.clone()
        got = M.gated_delta_step(**dict(a, v=v), state=second, slots=slots, out=v)
        assert got is v and torch.equal(v, want) and torch.equal(second, first)
        assert not strided or (wide[:, :8] == 3).all()


def test_arguments_and_result_in_one_buffer():
    a, state = arrays(40, 2, 4, 64, 48, torch.bfloat16)
    sizes = [2 * 64, 2 * 64, 4 * 48, 4 * 48]
    buffer = torch.zeros(40, sum(sizes), dtype=torch.bfloat16, device="cuda")
    q, k, v, y = buffer.split(sizes, 1)
    views = dict(q=q.view(40, 2, 64), k=k.view(40, 2, 64), v=v.view(40, 4, 48))
    for n, x in views.items():
        x.copy_(a[n])
    first, second = state.clone(), state.clone()
    want = M.gated_delta_step(**a, state=first)
    M.gated_delta_step(**dict(a, **views), state=second, out=y.view(40, 4, 48))
    assert torch.equal(y.reshape(40, 4, 48), want) and torch.equal(second, first)
    assert all(torch.equal(x, a[n]) for n, x in views.items())


@pytest.mark.parametrize("n", ["q", "k"])
def test_the_result_in_the_place_of_a_key_is_refused(n):
    a, state = arrays(40, 4, 4, 48, 48, torch.float32)
    before = {m: x.clone() for m, x in a.items()}
    with pytest.raises(M.MergesimError, match="overlap"):
        M.gated_delta_step(**a, state=state, out=a[n])
    assert all(torch.equal(a[m], x) for m, x in before.items())
