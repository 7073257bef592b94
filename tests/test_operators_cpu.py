"""The operators on device arrays on a machine without a GPU: what they refuse, and the sizes they name, come
from the host alone.  No pointer here is read: every call ends before it touches a GPU."""
import ctypes as C

import pytest
import torch  # noqa: F401  (before the library: both share one HIP runtime)

from paper_1805_11144_amd import mergesim as MS

A = 1 << 20   # an aligned address that nothing reads


def embed(**kw):
    d = MS.EmbedDesc(n_tokens=4, vocab=10, dim=8, scale=1.0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def gated(**kw):
    d = MS.GatedLowpassDesc(batch=2, steps=70000, dim=8)
    for k, v in kw.items():
        if k.endswith("stride"):
            getattr(d, k)[0], getattr(d, k)[1] = v
        else:
            setattr(d, k, v)
    return d


def step(**kw):
    d = MS.GatedStepDesc(rows=2, n_slots=4, dim=8)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def orth(**kw):
    d = MS.OrthDesc(batch=2, rows=8, cols=6, eps=1e-7, steps=5)
    d.coef[0], d.coef[1], d.coef[2] = kw.pop("coef", (3.4445, -4.7750, 2.0315))
    for k, v in kw.items():
        if k.endswith("stride"):
            getattr(d, k)[0], getattr(d, k)[1] = v
        else:
            setattr(d, k, v)
    return d


def refused(call, *args, words=""):
    lib = MS.load_library()
    code = getattr(lib, call)(*args)
    msg = lib.ms_last_error().decode()
    assert code == -1, (call, code, msg)
    assert words in msg, (call, msg)


@pytest.mark.parametrize("kw,words", [
    (dict(n_tokens=-1), "n_tokens"), (dict(n_tokens=1 << 31), "n_tokens"), (dict(vocab=0), "vocab"),
    (dict(vocab=1 << 31), "vocab"), (dict(dim=0), "dim"), (dict(dtype=2), "dtype"), (dict(grad_dtype=-1), "dtype"),
    (dict(ids=2), "token type"), (dict(scale=float("inf")), "scale"), (dict(table_stride=7), "strides"),
    (dict(row_stride=-8), "strides")])
def test_table_refusals(kw, words):
    refused("ms_embed", embed(**kw), A, A, A, words=words)
    refused("ms_embed_grad", embed(**kw), A, A, A, A, 1 << 30, words=words)
    refused("ms_embed_grad_workspace", embed(**kw), C.byref(C.c_int64()), words=words)


def test_table_pointer_and_workspace_refusals():
    for args in ((None, A, A), (A, None, A), (A, A, None)):
        refused("ms_embed", embed(), *args, words="NULL")
        refused("ms_embed_grad", embed(), *args, A, 1 << 30, words="NULL")
    refused("ms_embed", None, A, A, A, words="NULL")
    refused("ms_embed", embed(), A + 2, A, A, words="tokens")
    refused("ms_embed", embed(ids=1), A + 4, A, A, words="tokens")
    refused("ms_embed", embed(), A, A + 2, A, words="table")
    refused("ms_embed_grad", embed(dtype=1, grad_dtype=0), A, A + 2, A + 2, A, 1 << 30, words="dtable")
    n = C.c_int64()
    assert MS.load_library().ms_embed_grad_workspace(embed(), C.byref(n)) == 0 and n.value > 0
    refused("ms_embed_grad", embed(), A, A, A, None, n.value, words="workspace")
    refused("ms_embed_grad", embed(), A, A, A, A + 4, n.value, words="256")
    refused("ms_embed_grad", embed(), A, A, A, A, n.value - 1, words="too small")
    refused("ms_embed_grad_workspace", embed(), None, words="NULL")


@pytest.mark.parametrize("kw,words", [
    (dict(steps=-1), "steps"), (dict(steps=1 << 31), "steps"), (dict(dim=0), "dim"), (dict(batch=-1), "batch"),
    (dict(batch=1 << 30), "batch"), (dict(dtype=3), "dtype"), (dict(v_stride=(-8, 8)), "strides"),
    (dict(g_stride=(8, -8)), "strides")])
def test_gated_refusals(kw, words):
    refused("ms_gated_lowpass", gated(**kw), A, A, A, A, A, A, A, A, 1 << 30, words=words)
    refused("ms_gated_lowpass_grad", gated(**kw), A, A, A, A, A, A, A, A, A, A, 1 << 30, words=words)
    refused("ms_gated_lowpass_workspace", gated(**kw), C.byref(C.c_int64()), words=words)
    refused("ms_gated_lowpass_kept", gated(**kw), C.byref(C.c_int64()), words=words)


def test_gated_pointer_and_workspace_refusals():
    n = C.c_int64()
    assert MS.load_library().ms_gated_lowpass_workspace(gated(), C.byref(n)) == 0 and n.value > 0
    ok = [A, A, A, A, A, A, A, A, n.value]
    for i in (0, 1, 4):
        refused("ms_gated_lowpass", gated(), *[None if k == i else p for k, p in enumerate(ok)], words="NULL")
    refused("ms_gated_lowpass", gated(), *ok[:7], None, n.value, words="workspace")
    refused("ms_gated_lowpass", gated(), *ok[:8], n.value - 1, words="too small")
    refused("ms_gated_lowpass", gated(), A + 2, *ok[1:], words="aligned")
    refused("ms_gated_lowpass", gated(), A, A, A + 2, *ok[3:], words="aligned")
    refused("ms_gated_lowpass", gated(y_stride=(8, 4)), *ok, words="overlap")
    refused("ms_gated_lowpass", gated(y_stride=(4, 16)), *ok, words="overlap")
    ok = [A] * 10 + [n.value]
    for i in (0, 1, 2, 4, 6, 7):
        refused("ms_gated_lowpass_grad", gated(), *[None if k == i else p for k, p in enumerate(ok)], words="NULL")
    refused("ms_gated_lowpass_grad", gated(), *ok[:10], n.value - 1, words="too small")


@pytest.mark.parametrize("kw,words", [
    (dict(rows=-1), "rows"), (dict(n_slots=-1), "n_slots"), (dict(dim=0), "dim"), (dict(dtype=7), "dtype"),
    (dict(v_stride=4), "strides"), (dict(state_stride=-8), "strides")])
def test_step_refusals(kw, words):
    refused("ms_gated_lowpass_step", step(**kw), A, A, A, A, A, words=words)


def test_step_pointer_refusals():
    for args in ((None, A, A, A, A), (A, None, A, A, A), (A, A, None, A, A), (A, A, A, A, None)):
        refused("ms_gated_lowpass_step", step(), *args, words="NULL")
    refused("ms_gated_lowpass_step", step(), A, A, A + 2, A, A, words="aligned")


@pytest.mark.parametrize("kw,words", [
    (dict(rows=0), "rows"), (dict(cols=65537), "cols"), (dict(batch=-1), "batch"), (dict(batch=1 << 40), "too many"),
    (dict(steps=0), "steps"), (dict(steps=101), "steps"), (dict(dtype=2), "dtype"), (dict(eps=-1.0), "eps"),
    (dict(eps=float("nan")), "eps"), (dict(coef=(2.0, 1.0, 1.0)), "grow"), (dict(coef=(float("nan"), 0, 0)), "finite"),
    (dict(coef=(2000.0, 0, 0)), "grow"), (dict(x_stride=(48, 5)), "strides"), (dict(out_stride=(-1, 6)), "strides")])
def test_orth_refusals(kw, words):
    refused("ms_orthogonalise", orth(**kw), A, A, A, 1 << 40, words=words)
    refused("ms_orthogonal_update", orth(**kw), MS.OrthRule(0.1, 0.9, 0.0, 1), A, A, A, A, 1 << 40, words=words)
    refused("ms_orth_workspace", orth(**kw), 0, C.byref(C.c_int64()), words=words)


def test_orth_pointer_and_rule_refusals():
    rule = MS.OrthRule(0.1, 0.9, 0.0, 1)
    refused("ms_orthogonalise", orth(), None, A, A, 1 << 40, words="NULL")
    refused("ms_orthogonalise", orth(), A, None, A, 1 << 40, words="NULL")
    refused("ms_orthogonalise", orth(), A + 2, A, A, 1 << 40, words="aligned")
    refused("ms_orthogonalise", orth(out_stride=(40, 6)), A, A, A, 1 << 40, words="overlap")
    big = orth(rows=1000, cols=900)   # past the sizes that need no workspace, if there are any
    refused("ms_orthogonalise", big, A, A, A, 16, words="too small")
    refused("ms_orthogonal_update", orth(), None, A, A, A, A, 1 << 40, words="rule")
    refused("ms_orthogonal_update", orth(), MS.OrthRule(float("inf"), 0.9, 0.0, 1), A, A, A, A, 1 << 40, words="finite")
    for args in ((None, A, A), (A, None, A), (A, A, None)):
        refused("ms_orthogonal_update", orth(), rule, *args, A, 1 << 40, words="NULL")


def test_many_small_matrices_need_no_workspace():
    n = C.c_int64(-1)
    assert MS.load_library().ms_orth_workspace(orth(batch=1 << 20), 0, C.byref(n)) == 0 and n.value == 0
    refused("ms_orth_workspace", orth(batch=1 << 20, rows=500, cols=400), 0, C.byref(n), words="too many")


def test_empty_calls_succeed_without_a_gpu():
    lib = MS.load_library()
    assert lib.ms_embed(embed(n_tokens=0), None, None, None) == 0
    assert lib.ms_gated_lowpass(gated(batch=0), None, None, None, None, None, None, None, None, 0) == 0
    assert lib.ms_gated_lowpass_step(step(rows=0), None, None, None, None, None) == 0
    assert lib.ms_orthogonalise(orth(batch=0), None, None, None, 0) == 0


def test_the_binding_refuses_arrays_of_the_host():
    import paper_1805_11144_amd as M
    x = torch.zeros(3, 4)
    for call in (lambda: M.embed(torch.zeros(2, dtype=torch.int32), x), lambda: M.orthogonalise(x),
                 lambda: M.embed_grad(torch.zeros(3, dtype=torch.int32), x, 5),
                 lambda: M.gated_lowpass(x[None], x[None]), lambda: M.gated_lowpass_step(x, x, x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
