"""The library's operators on GPU arrays (include/mergesim.h, "operators on device arrays"): marshalling only.

Arrays are torch tensors on one GPU; a call runs on that GPU's current torch stream, allocates its
results and scratch memory with torch and returns without waiting, so it can be captured into a graph.
torch has to be imported before the library is first used in a process, so that both share one HIP
runtime.
"""
from __future__ import annotations

import ctypes as C

from . import mergesim as _ms
from .mergesim import (DTYPE_BF16, DTYPE_F32, IDS_I32, IDS_I64, EmbedDesc, GatedLowpassDesc, GatedStepDesc, OrthDesc,
                       OrthRule, _check)

NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)   # raises small singular values fast; leaves them within 0.3 of one

_state = {}


def _setup():
    """(torch, library): checked once that they share one HIP runtime."""
    if not _state:
        import torch
        lib = _ms.load_library()
        with open("/proc/self/maps") as f:
            runtimes = {line.split()[-1] for line in f if "libamdhip64" in line}
        if len(runtimes) > 1:
            raise ImportError("the library was loaded with another HIP runtime than torch's: import torch first "
                              f"({', '.join(sorted(runtimes))})")
        _state["dtypes"] = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}
        _state["ids"] = {torch.int32: IDS_I32, torch.int64: IDS_I64}
        _state["both"] = torch, lib
    return _state["both"]


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _dtype(t, name):
    d = _state["dtypes"].get(t.dtype)
    _need(d is not None, f"{name} is {t.dtype}: float32 or bfloat16 is wanted")
    return d


def _like(t, first, name, shape=None, dtype=None):
    """Checks a tensor's device, and its shape and type where given."""
    _need(t.is_cuda and t.device == first.device, f"{name} must be on the GPU of the other arrays ({first.device})")
    _need(shape is None or tuple(t.shape) == tuple(shape), f"{name} has shape {tuple(t.shape)}, not {shape}")
    _need(dtype is None or t.dtype == dtype, f"{name} is {t.dtype}, not {dtype}")


def _packed(t, name):
    _need(t.is_contiguous(), f"{name} must be contiguous")
    return t.data_ptr()


def _on(d, t, torch):
    """The descriptor's device and stream: torch's current one there."""
    d.device = t.device.index
    d.stream = torch.cuda.current_stream(t.device).cuda_stream
    return C.byref(d)


def _row_stride(t, name):
    """Elements between the rows of a matrix [n, dim] whose rows are contiguous."""
    n, dim = t.shape
    _need(dim == 1 or t.stride(1) == 1, f"{name}'s rows must be contiguous")
    if n <= 1:
        return dim
    _need(t.stride(0) >= dim, f"{name}'s rows overlap")
    return t.stride(0)


def _scratch(torch, like, call, *args):
    """Scratch memory of the size that `call` names."""
    n = C.c_int64()
    _check(call(*args, C.byref(n)))
    if n.value == 0:
        return None, None, 0
    w = torch.empty(n.value, dtype=torch.uint8, device=like.device)
    return w, w.data_ptr(), n.value


# ------------------------------------------------------------------------ tables
def _embed_desc(torch, tokens, rows, table_stride, row_stride, vocab, scale):
    d = EmbedDesc()
    ids = _state["ids"].get(tokens.dtype)
    _need(ids is not None, f"tokens are {tokens.dtype}: int32 or int64 is wanted")
    d.n_tokens, d.vocab, d.dim = tokens.numel(), vocab, rows.shape[-1]
    d.table_stride, d.row_stride, d.scale, d.ids, d.dtype = table_stride, row_stride, scale, ids, _dtype(rows, "rows")
    return d


def embed(tokens, table, scale=1.0, out=None):
    """out[..., :] = scale * table[tokens[...], :], zeros for tokens outside the table (ms_embed).

    tokens: int32 or int64 of any shape; table [vocab, dim] float32 or bfloat16."""
    torch, lib = _setup()
    _need(table.is_cuda and table.dim() == 2, "table must be a matrix on a GPU")
    _like(tokens, table, "tokens")
    tokens = tokens.contiguous()
    shape = (*tokens.shape, table.shape[1])
    if out is None:
        out = torch.empty(shape, dtype=table.dtype, device=table.device)
    _like(out, table, "out", shape, table.dtype)
    d = _embed_desc(torch, tokens, table, _row_stride(table, "table"), 0, table.shape[0], scale)
    _check(lib.ms_embed(_on(d, table, torch), tokens.data_ptr(), table.data_ptr(), _packed(out, "out")))
    return out


def embed_grad(tokens, drows, vocab=None, scale=1.0, out=None, accumulate=False):
    """The gradient [vocab, dim] of `embed`'s table (ms_embed_grad): for each token, scale times the sum of its
    rows of drows [*tokens.shape, dim], in an order that depends on the tokens alone.

    float32, or the type of `out`; accumulate: added to what `out` holds."""
    torch, lib = _setup()
    _need(drows.is_cuda and drows.dim() >= 1, "drows must be on a GPU")
    dim = drows.shape[-1]
    _like(drows, drows, "drows", (*tokens.shape, dim))
    _like(tokens, drows, "tokens")
    _need(out is not None or not accumulate, "accumulate needs out")
    if out is None:
        _need(vocab is not None, "vocab or out is wanted")
        out = torch.empty((vocab, dim), dtype=torch.float32, device=drows.device)
    _like(out, drows, "out", (out.shape[0] if vocab is None else vocab, dim))
    tokens, rows = tokens.contiguous(), drows.reshape(-1, dim)
    if rows.shape[0] > 1 and (rows.stride(0) < dim or (dim > 1 and rows.stride(1) != 1)):
        rows = rows.contiguous()   # a broadcast gradient
    d = _embed_desc(torch, tokens, rows, _row_stride(out, "out"), _row_stride(rows, "drows"), out.shape[0], scale)
    d.grad_dtype, d.accumulate = _dtype(out, "out"), int(bool(accumulate))
    ref = _on(d, drows, torch)
    keep, ws, n = _scratch(torch, drows, lib.ms_embed_grad_workspace, ref)
    _check(lib.ms_embed_grad(ref, tokens.data_ptr(), rows.data_ptr(), out.data_ptr(), ws, n))
    return out


# ----------------------------------------------------------------- gated lowpass
def _sequence(t, name):
    """(tensor, [batch stride, step stride]) of [batch, steps, dim] with contiguous channels."""
    batch, steps, dim = t.shape
    _need(dim >= 1, f"{name} has no channels")
    sb, ss = t.stride(0) if batch > 1 else 0, t.stride(1) if steps > 1 else 0
    if (dim > 1 and t.stride(2) != 1) or (batch * steps > 1 and sb == ss == 0):
        t = t.contiguous()
        sb = ss = 0
    return t, (sb, ss)


def _gated_desc(v, g, y):
    _need(v.is_cuda and v.dim() == 3, "v must be [batch, steps, dim] on a GPU")
    _like(g, v, "g", v.shape, v.dtype)
    d = GatedLowpassDesc()
    d.batch, d.steps, d.dim = v.shape
    d.dtype = _dtype(v, "v")
    v, (d.v_stride[0], d.v_stride[1]) = _sequence(v, "v")
    g, (d.g_stride[0], d.g_stride[1]) = _sequence(g, "g")
    y, (d.y_stride[0], d.y_stride[1]) = _sequence(y, "y")
    return d, v, g, y


def _optional(torch, t, v, name, shape, dtype):
    if t is None:
        return None
    _like(t, v, name, shape, dtype)
    return _packed(t, name)


def gated_lowpass(v, g, y0=None, lengths=None, keep=False):
    """The lowpass synapse whose coefficient the input sets (ms_gated_lowpass): with a = sigmoid(g),
    y[:, t] = a[:, t] y[:, t-1] + (1 - a[:, t]) v[:, t] from y0 (zeros).

    v, g [batch, steps, dim], float32 or bfloat16; y0 [batch, dim] float32; lengths int32 [batch].
    Returns (y, last): y like v, zeros past a row's length, and the state after its last step, float32.
    keep: also the states that gated_lowpass_grad starts from."""
    torch, lib = _setup()
    _need(v.is_cuda and v.dim() == 3, "v must be [batch, steps, dim] on a GPU")
    batch, steps, dim = v.shape
    y = torch.empty((batch, steps, dim), dtype=v.dtype, device=v.device)
    last = torch.empty((batch, dim), dtype=torch.float32, device=v.device)
    d, v, g, y = _gated_desc(v, g, y)
    ref = _on(d, v, torch)
    kept = None
    if keep:
        n = C.c_int64()
        _check(lib.ms_gated_lowpass_kept(ref, C.byref(n)))
        kept = torch.empty(n.value, dtype=torch.float32, device=v.device)
    hold, ws, n = _scratch(torch, v, lib.ms_gated_lowpass_workspace, ref)
    _check(lib.ms_gated_lowpass(ref, v.data_ptr(), g.data_ptr(),
                                _optional(torch, y0, v, "y0", (batch, dim), torch.float32),
                                _optional(torch, lengths, v, "lengths", (batch,), torch.int32),
                                y.data_ptr(), last.data_ptr(), None if kept is None else kept.data_ptr(), ws, n))
    return (y, last, kept) if keep else (y, last)


def gated_lowpass_grad(v, g, kept, dy, dlast=None, lengths=None):
    """(dv, dg, dy0) of gated_lowpass from dL/dy and dL/dlast (ms_gated_lowpass_grad); kept: what the forward
    call with keep=True left."""
    torch, lib = _setup()
    _need(v.is_cuda and v.dim() == 3, "v must be [batch, steps, dim] on a GPU")
    _like(dy, v, "dy", v.shape, v.dtype)
    batch, steps, dim = v.shape
    dv = torch.empty((batch, steps, dim), dtype=v.dtype, device=v.device)
    dg = torch.empty_like(dv)
    dy0 = torch.empty((batch, dim), dtype=torch.float32, device=v.device)
    d, v, g, dy = _gated_desc(v, g, dy)
    ref = _on(d, v, torch)
    n = C.c_int64()
    _check(lib.ms_gated_lowpass_kept(ref, C.byref(n)))
    _like(kept, v, "kept", (n.value,), torch.float32)
    hold, ws, n = _scratch(torch, v, lib.ms_gated_lowpass_workspace, ref)
    _check(lib.ms_gated_lowpass_grad(ref, v.data_ptr(), g.data_ptr(), _packed(kept, "kept"),
                                     _optional(torch, lengths, v, "lengths", (batch,), torch.int32), dy.data_ptr(),
                                     _optional(torch, dlast, v, "dlast", (batch, dim), torch.float32),
                                     dv.data_ptr(), dg.data_ptr(), dy0.data_ptr(), ws, n))
    return dv, dg, dy0


def gated_lowpass_step(v, g, state, slots=None, out=None):
    """One step for the sequences being served (ms_gated_lowpass_step): row i of v, g [rows, dim] advances
    state[slots[i]] (float32 [slots, dim], in place; row i's own slot without `slots`, int32) and returns it in
    v's type; a slot outside the cache marks an idle row, whose result is zeros."""
    torch, lib = _setup()
    _need(v.is_cuda and v.dim() == 2, "v must be [rows, dim] on a GPU")
    rows, dim = v.shape
    _like(g, v, "g", v.shape, v.dtype)
    _like(state, v, "state", (state.shape[0], dim), torch.float32)
    if out is None:
        out = torch.empty((rows, dim), dtype=v.dtype, device=v.device)
    _like(out, v, "out", v.shape, v.dtype)
    d = GatedStepDesc()
    d.rows, d.n_slots, d.dim, d.dtype = rows, state.shape[0], dim, _dtype(v, "v")
    d.v_stride, d.g_stride = _row_stride(v, "v"), _row_stride(g, "g")
    d.y_stride, d.state_stride = _row_stride(out, "out"), _row_stride(state, "state")
    _check(lib.ms_gated_lowpass_step(_on(d, v, torch), v.data_ptr(), g.data_ptr(), state.data_ptr(),
                                     _optional(torch, slots, v, "slots", (rows,), torch.int32), out.data_ptr()))
    return out


# ---------------------------------------------------------- orthogonalised updates
def _orth_desc(x, steps, coefficients, eps):
    _need(x.is_cuda and x.dim() in (2, 3), "a matrix or a batch of matrices on a GPU is wanted")
    d = OrthDesc()
    rows, cols = x.shape[-2:]
    batch = x.shape[0] if x.dim() == 3 else 1
    if (cols > 1 and x.stride(-1) != 1) or (rows > 1 and x.stride(-2) < cols):
        x = x.contiguous()
    d.batch, d.rows, d.cols = batch, rows, cols
    d.x_stride[1] = x.stride(-2) if rows > 1 else cols
    d.x_stride[0] = x.stride(0) if x.dim() == 3 and batch > 1 else 0
    d.coef[0], d.coef[1], d.coef[2] = coefficients
    d.eps, d.steps, d.dtype = eps, steps, _dtype(x, "x")
    return d, x


def orthogonalise(x, steps=5, coefficients=NEWTON_SCHULZ, eps=1e-7, out=None):
    """Brings the singular values of a matrix [rows, cols], or of each of a batch, towards one
    (ms_orthogonalise): X <- (c0 I + c1 XX' + c2 XX'XX') X, `steps` times from X / (|X| + eps)."""
    torch, lib = _setup()
    d, x = _orth_desc(x, steps, coefficients, eps)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _like(out, x, "out", x.shape, x.dtype)
    ref = _on(d, x, torch)
    hold, ws, n = _scratch(torch, x, lib.ms_orth_workspace, ref, 0)
    _check(lib.ms_orthogonalise(ref, x.data_ptr(), _packed(out, "out"), ws, n))
    return out


def orthogonal_update(weight, momentum, grad, rate, momentum_decay=0.95, weight_decay=0.0, nesterov=True, steps=5,
                      coefficients=NEWTON_SCHULZ, eps=1e-7):
    """One training step of a weight matrix, or a batch of them (ms_orthogonal_update), in place: momentum <-
    momentum_decay momentum + grad; weight <- (1 - rate weight_decay) weight - rate orthogonalise(grad +
    momentum_decay momentum), or of the momentum alone without nesterov.

    weight, momentum: float32, contiguous; grad: float32 or bfloat16."""
    torch, lib = _setup()
    d, grad = _orth_desc(grad, steps, coefficients, eps)
    _like(weight, grad, "weight", grad.shape, torch.float32)
    _like(momentum, grad, "momentum", grad.shape, torch.float32)
    rule = OrthRule(rate, momentum_decay, weight_decay, int(bool(nesterov)))
    ref = _on(d, grad, torch)
    hold, ws, n = _scratch(torch, grad, lib.ms_orth_workspace, ref, 1)
    _check(lib.ms_orthogonal_update(ref, C.byref(rule), _packed(weight, "weight"), _packed(momentum, "momentum"),
                                    grad.data_ptr(), ws, n))
