"""What the binding of the gated delta rule's step hands to the library as the cache of matrices, with the library's call
replaced: nothing here runs on a GPU.  Every matrix that the descriptor names has to lie in the array's own memory."""
import pytest
import torch

import paper_1805_11144_amd.operators as O
from paper_1805_11144_amd import mergesim as MS

HEADS, KEYS, VALUES = 2, 4, 6
MATRICES = HEADS * KEYS * VALUES


@pytest.fixture
def calls(monkeypatch):
    seen = []

    class Library:
        @staticmethod
        def ms_gated_delta_step(d, q, k, v, decay, rate, state, slots, out):
            seen.append((d, state))
            return 0
    monkeypatch.setattr(O, "_torch", torch)
    monkeypatch.setattr(O, "_forward", torch.autograd.forward_ad)
    monkeypatch.setattr(O, "_lib", Library)
    monkeypatch.setattr(O, "_gpu", lambda t, dims, what: MS.DTYPE_F32)
    monkeypatch.setattr(O, "_on", lambda d, t: d)
    return seen


def step(state, rows=2):
    f = torch.zeros
    return O.gated_delta_step(f(rows, 1, KEYS), f(rows, 1, KEYS), f(rows, HEADS, VALUES), f(rows, HEADS), f(rows, HEADS), state)


def addressed(d, state, address):
    """The first and one past the last value that the library may write, of the storage's own."""
    stride = d.state_stride or MATRICES
    first = (address - state.untyped_storage().data_ptr()) // 4
    return first, first + (d.n_slots - 1) * stride + MATRICES


@pytest.mark.parametrize("state", [
    torch.zeros(3, HEADS, KEYS, VALUES), torch.zeros(1, HEADS, KEYS, VALUES),
    torch.zeros(5, HEADS, KEYS, VALUES)[1:4], torch.zeros(6, HEADS, KEYS, VALUES)[::2],
    torch.zeros(3, 2, HEADS, KEYS, VALUES)[:, 1], torch.zeros(1, HEADS, KEYS, VALUES).expand(1, -1, -1, -1)])
def test_matrices_lie_in_the_array(calls, state):
    step(state)
    (d, address), = calls
    first, last = addressed(d, state, address)
    assert d.n_slots == state.shape[0] and address == state.data_ptr()
    assert 0 <= first and last <= state.untyped_storage().nbytes() // 4


@pytest.mark.parametrize("state", [
    torch.zeros(1, HEADS, KEYS, VALUES).expand(4, -1, -1, -1), torch.zeros(HEADS, KEYS, VALUES).expand(2, -1, -1, -1),
    torch.zeros(4 * MATRICES).as_strided((4, HEADS, KEYS, VALUES), (MATRICES // 2, KEYS * VALUES, VALUES, 1)),
    torch.zeros(4 * MATRICES).as_strided((4, HEADS, KEYS, VALUES), (MATRICES - 1, KEYS * VALUES, VALUES, 1))])
def test_slots_that_share_memory_are_refused(calls, state):
    with pytest.raises(ValueError, match="overlap"):
        step(state)
    assert not calls


@pytest.mark.parametrize("state", [
    torch.zeros(4, KEYS, HEADS, VALUES).transpose(1, 2), torch.zeros(4, HEADS, KEYS, 2 * VALUES)[..., ::2],
    torch.zeros(4, HEADS, KEYS, 2 * VALUES)[..., :VALUES], torch.zeros(4, 1, KEYS, VALUES).expand(4, HEADS, KEYS, VALUES)])
def test_matrices_that_are_not_packed_are_refused(calls, state):
    with pytest.raises(ValueError, match="contiguous"):
        step(state)
    assert not calls
