"""The operators of keyed memories (gated delta rule, group norm) on a machine without a GPU: what they refuse, and the
sizes they name, come from the host alone.  No pointer here is read: every call ends before it touches a GPU."""
import ctypes as C

import pytest
import torch  # noqa: F401  (before the library: both share one HIP runtime)

from paper_1805_11144_amd import mergesim as MS
from test_operators_cpu import A, refused


def filled(d, kw):
    for k, v in kw.items():
        if k.endswith("stride") and isinstance(v, tuple):
            getattr(d, k)[:] = v
        else:
            setattr(d, k, v)
    return d


def delta(**kw):
    return filled(MS.GatedDeltaDesc(batch=2, steps=100, heads=4, key_heads=2, keys=24, values=40, scale=1.0), kw)


def step(**kw):
    return filled(MS.GatedDeltaStepDesc(rows=2, n_slots=4, heads=4, key_heads=2, keys=24, values=40, scale=1.0), kw)


def norm(**kw):
    return filled(MS.GroupNormDesc(batch=2, positions=50, channels=24, groups=4, eps=1e-5), kw)


def size(call, *args):
    n = C.c_int64(-1)
    assert getattr(MS.load_library(), call)(*args, C.byref(n)) == 0
    return n.value


BIG = 1 << 40


@pytest.mark.parametrize("kw,words", [
    (dict(steps=-1), "steps"), (dict(steps=1 << 31), "steps"), (dict(batch=-1), "batch"), (dict(batch=1 << 31), "batch"),
    (dict(heads=0), "heads"), (dict(key_heads=0), "heads"), (dict(key_heads=3), "heads"), (dict(heads=65538), "heads"),
    (dict(keys=0), "keys"), (dict(keys=129), "keys"), (dict(values=0), "values"), (dict(values=65537), "values"),
    (dict(dtype=2), "dtype"), (dict(scale=float("nan")), "scale"), (dict(scale=1e300), "scale"),
    (dict(q_stride=(-1, 1, 1)), "strides"), (dict(k_stride=(1, -1, 1)), "strides"), (dict(v_stride=(1, 1, -1)), "strides"),
    (dict(decay_stride=(-8, 8, 1)), "strides"), (dict(rate_stride=(8, 1 << 40, 1)), "strides"),
    (dict(heads=1024, values=16384), "2^24"), (dict(v_stride=(1, 1 << 24, 1)), "2^24"), (dict(y_stride=(1, 1 << 24, 1)), "2^24"),
    (dict(batch=1 << 22), "too large"), (dict(batch=1 << 20, steps=1 << 30), "too large")])
def test_delta_refusals(kw, words):
    refused("ms_gated_delta", delta(**kw), *[A] * 11, BIG, words=words)
    refused("ms_gated_delta_grad", delta(**kw), *[A] * 16, BIG, words=words)
    refused("ms_gated_delta_workspace", delta(**kw), 0, C.byref(C.c_int64()), words=words)
    refused("ms_gated_delta_kept", delta(**kw), C.byref(C.c_int64()), words=words)


def test_delta_pointer_and_workspace_refusals():
    n = size("ms_gated_delta_workspace", delta(), 0)
    ok = [A] * 11 + [n]
    for i in (0, 1, 2, 3, 4, 7):
        refused("ms_gated_delta", delta(), *[None if k == i else p for k, p in enumerate(ok)], words="NULL")
        refused("ms_gated_delta", delta(), *[A + 2 if k == i else p for k, p in enumerate(ok)], words="aligned")
    for i in (5, 6, 8, 9):
        refused("ms_gated_delta", delta(), *[A + 2 if k == i else p for k, p in enumerate(ok)], words="aligned")
    refused("ms_gated_delta", None, *ok, words="NULL")
    refused("ms_gated_delta", delta(), *ok[:10], None, n, words="workspace")
    refused("ms_gated_delta", delta(), *ok[:10], A + 16, n, words="256")
    refused("ms_gated_delta", delta(), *ok[:11], n - 1, words="too small")
    for y in ((16000, 160, 39), (16000, 159, 40), (15999, 160, 40), (16000, 40, 40), (0, 160, 40)):
        refused("ms_gated_delta", delta(y_stride=y), *ok, words="overlap")
    n = size("ms_gated_delta_workspace", delta(), 1)
    ok = [A] * 16 + [n]
    for i in (0, 1, 2, 3, 4, 5, 7, 9, 10, 11, 12, 13):
        refused("ms_gated_delta_grad", delta(), *[None if k == i else p for k, p in enumerate(ok)], words="NULL")
        refused("ms_gated_delta_grad", delta(), *[A + 2 if k == i else p for k, p in enumerate(ok)], words="aligned")
    for i in (6, 8, 14):
        refused("ms_gated_delta_grad", delta(), *[A + 2 if k == i else p for k, p in enumerate(ok)], words="aligned")
    refused("ms_gated_delta_grad", delta(), *ok[:16], n - 1, words="too small")
    refused("ms_gated_delta_workspace", delta(), 0, None, words="NULL")
    refused("ms_gated_delta_kept", delta(), None, words="NULL")


@pytest.mark.parametrize("kw,words", [
    (dict(rows=-1), "rows"), (dict(n_slots=1 << 31), "n_slots"), (dict(heads=3), "heads"), (dict(keys=129), "keys"),
    (dict(values=0), "values"), (dict(dtype=7), "dtype"), (dict(scale=float("inf")), "scale"),
    (dict(q_stride=(-1, 1)), "strides"), (dict(state_stride=3839), "strides"), (dict(y_stride=(159, 40)), "overlap"),
    (dict(y_stride=(160, 39)), "overlap")])
def test_delta_step_refusals(kw, words):
    refused("ms_gated_delta_step", step(**kw), *[A] * 8, words=words)


def test_delta_step_pointer_refusals():
    ok = [A] * 8
    for i in (0, 1, 2, 3, 4, 5, 7):
        refused("ms_gated_delta_step", step(), *[None if k == i else p for k, p in enumerate(ok)], words="NULL")
    for i in range(8):
        refused("ms_gated_delta_step", step(), *[A + 2 if k == i else p for k, p in enumerate(ok)], words="aligned")


@pytest.mark.parametrize("kw,words", [
    (dict(batch=-1), "batch"), (dict(positions=1 << 31), "positions"), (dict(channels=0), "channels"),
    (dict(channels=1 << 24, groups=1), "channels"), (dict(groups=0), "channels"), (dict(groups=5), "channels"),
    (dict(dtype=2), "dtype"), (dict(activation=3), "activation"), (dict(activation=-1), "activation"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=1e300), "eps"), (dict(x_stride=(-1, 24)), "strides"),
    (dict(y_stride=(24, -1)), "strides"), (dict(batch=(1 << 31) - 1, channels=(1 << 24) - 4), "too large")])
def test_norm_refusals(kw, words):
    refused("ms_group_norm", norm(**kw), *[A] * 7, BIG, words=words)
    refused("ms_group_norm_grad", norm(**kw), *[A] * 10, BIG, words=words)
    refused("ms_group_norm_workspace", norm(**kw), 0, C.byref(C.c_int64()), words=words)


def test_norm_pointer_and_workspace_refusals():
    big = dict(positions=5000)
    n = size("ms_group_norm_workspace", norm(**big), 0)
    assert n > 0
    ok = [A] * 7 + [n]
    for i in (0, 4):
        refused("ms_group_norm", norm(**big), *[None if k == i else p for k, p in enumerate(ok)], words="NULL")
    for i in range(6):
        refused("ms_group_norm", norm(**big), *[A + 2 if k == i else p for k, p in enumerate(ok)],
                words="aligned" if i not in (0, 4) else "")
    refused("ms_group_norm", norm(**big), *ok[:6], None, n, words="workspace")
    refused("ms_group_norm", norm(**big), *ok[:7], n - 1, words="too small")
    refused("ms_group_norm", norm(y_stride=(24, 12)), *ok, words="overlap")
    n = size("ms_group_norm_workspace", norm(), 1)
    ok = [A] * 10 + [n]
    for i in (0, 4, 5, 6, 7, 8):
        refused("ms_group_norm_grad", norm(), *[None if k == i else p for k, p in enumerate(ok)], words="NULL")
    refused("ms_group_norm_grad", norm(), *ok[:10], n - 1, words="too small")
    refused("ms_group_norm_workspace", norm(), 0, None, words="NULL")


def test_empty_calls():
    lib = MS.load_library()
    assert lib.ms_gated_delta(delta(batch=0), *[None] * 11, 0) == 0
    assert lib.ms_gated_delta_grad(delta(batch=0), *[None] * 16, 0) == 0
    assert lib.ms_gated_delta_step(step(rows=0), *[None] * 8) == 0
    for d in (norm(batch=0), norm(positions=0)):
        assert lib.ms_group_norm(d, *[None] * 7, 0) == 0
    for grad in (0, 1):
        for d in (norm(batch=0), norm(positions=0), norm(batch=0, positions=0), norm(batch=0, positions=1)):
            assert size("ms_group_norm_workspace", d, grad) >= 0
        for d in (delta(batch=0), delta(steps=0)):
            assert size("ms_gated_delta_workspace", d, grad) == 0
    assert size("ms_gated_delta_kept", delta(steps=0)) == 0


def test_extreme_sizes_are_named_or_refused():
    for grad in (0, 1):
        for d in (norm(batch=1, positions=(1 << 31) - 1, channels=511, groups=1),
                  norm(batch=(1 << 16) - 1, positions=1, channels=(1 << 24) - 1, groups=(1 << 24) - 1),
                  norm(batch=(1 << 31) - 1, positions=(1 << 31) - 1, channels=1, groups=1)):
            assert 0 <= size("ms_group_norm_workspace", d, grad) < 1 << 62
        d = delta(batch=1, steps=(1 << 21) - 1, heads=8, key_heads=1, keys=128, values=65536, dtype=1)
        assert 0 < size("ms_gated_delta_workspace", d, grad) < 1 << 62


def test_the_binding_refuses_arrays_of_the_host():
    import paper_1805_11144_amd as M
    x, g, s = torch.zeros(2, 3, 4, 5), torch.zeros(2, 3, 4), torch.zeros(2, 4, 5, 5)
    for call in (lambda: M.gated_delta(x, x, x, g, g), lambda: M.gated_delta_grad(x, x, x, g, g, s, x),
                 lambda: M.gated_delta_step(x[0], x[0], x[0], g[0], g[0], s), lambda: M.group_norm(x, 5),
                 lambda: M.group_norm_grad(x, 5, s, x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
