"""The library's operators on GPU arrays (include/mergesim.h, "operators on device arrays"): marshalling only.

Arrays are torch tensors on one GPU; a call runs on that GPU's current torch stream, allocates its
results and scratch memory with torch and returns without waiting, so it can be captured into a graph.
torch has to be imported before the library is first used in a process, so that both share one HIP
runtime.

torch's automatic differentiation does not see these calls: an array that requires a gradient is refused
(outside torch.no_grad(), which is where a training step of one's own makes them), and an array that a call
writes in place counts as modified.
"""
from __future__ import annotations

import ctypes as C

from . import mergesim as _ms
from .mergesim import (DTYPE_BF16, DTYPE_F32, IDS_I32, IDS_I64, EmbedDesc, GatedLowpassDesc, GatedStepDesc, OrthDesc,
                       OrthRule, _check)

# Raises small singular values fast and leaves them within 0.3 of one: the coefficients published by K. Jordan et al.,
# "Muon: An optimizer for hidden layers in neural networks" (2024).
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)

_torch = _lib = _stream = None
_DTYPES, _IDS = {}, {}


def _setup():
    """Loads torch and the library, once, and checks that they share one HIP runtime."""
    global _torch, _lib, _stream
    import torch
    lib = _ms.load_library()
    with open("/proc/self/maps") as f:
        runtimes = {line.split()[-1] for line in f if "libamdhip64" in line}
    if len(runtimes) > 1:
        raise ImportError("the library was loaded with another HIP runtime than torch's: import torch first "
                          f"({', '.join(sorted(runtimes))})")
    _DTYPES.update({torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16})
    _IDS.update({torch.int32: IDS_I32, torch.int64: IDS_I64})
    # the current stream's handle without a Stream object around it: 2 of the 11 us of a small call
    _stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
    _torch, _lib = torch, lib


def _gpu(t, dims, what):
    if _lib is None:
        _setup()
    if not t.is_cuda or t.dim() not in dims:
        raise ValueError(f"{what} on a GPU is wanted, not {tuple(t.shape)} on {t.device}")
    _undifferentiated(t, what)
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"{what} is {t.dtype}: float32 or bfloat16 is wanted")
    return d


def _undifferentiated(t, what):
    if t.requires_grad and _torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient, which torch cannot take through this call: detach it, or call "
                         "under torch.no_grad() and use the operator's own gradient")


def _written(*tensors):
    """Tells torch that a call writes these, so that a backward pass which saved one raises."""
    for t in tensors:
        if t.is_inference() and not _torch.is_inference_mode_enabled():
            raise RuntimeError("an inference tensor can be written in place in torch.inference_mode() only")
    _torch.autograd.graph.increment_version(tensors)


def _like(t, first, name, shape, dtype):
    """Checks a tensor's device, shape and type."""
    _undifferentiated(t, name)
    if t.device != first.device:
        raise ValueError(f"{name} must be on the GPU of the other arrays ({first.device}), not on {t.device}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.dtype is not dtype:
        raise ValueError(f"{name} is {t.dtype}, not {dtype}")
    return t


def _packed(t, first, name, shape, dtype):
    """The address of a contiguous tensor, or None for None."""
    if t is None:
        return None
    if not _like(t, first, name, shape, dtype).is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _on(d, t):
    """The descriptor's device and stream: torch's current one there."""
    d.device = t.device.index
    d.stream = _stream(d.device)
    return C.byref(d)


def _row_stride(t, name):
    """Elements between the rows of a matrix [n, dim] whose rows are contiguous."""
    n, dim = t.shape
    rows, cols = t.stride()
    if dim > 1 and cols != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    if n <= 1:
        return dim
    if rows < dim:
        raise ValueError(f"{name}'s rows overlap")
    return rows


def _scratch(t, n):
    """(tensor, address, bytes) of n bytes of scratch memory on t's GPU."""
    if n == 0:
        return None, None, 0
    w = _torch.empty(n, dtype=_torch.uint8, device=t.device)
    return w, w.data_ptr(), n


def _size(call, *args):
    n = C.c_int64()
    _check(call(*args, C.byref(n)))
    return n.value


# ------------------------------------------------------------------------ tables
def _embed_desc(tokens, first):
    if tokens.device != first.device:
        raise ValueError(f"tokens must be on the GPU of the other arrays ({first.device}), not on {tokens.device}")
    ids = _IDS.get(tokens.dtype)
    if ids is None:
        raise ValueError(f"tokens are {tokens.dtype}: int32 or int64 is wanted")
    return EmbedDesc(n_tokens=tokens.numel(), ids=ids)


def embed(tokens, table, scale=1.0, out=None):
    """out[..., :] = scale * table[tokens[...], :], zeros for tokens outside the table (ms_embed).

    tokens: int32 or int64 of any shape; table [vocab, dim] float32 or bfloat16."""
    dtype = _gpu(table, (2,), "a table [vocab, dim]")
    d = _embed_desc(tokens, table)
    tokens = tokens.contiguous()
    shape = (*tokens.shape, table.shape[1])
    given = out is not None
    if not given:
        out = _torch.empty(shape, dtype=table.dtype, device=table.device)
    d.vocab, d.dim = table.shape
    d.table_stride, d.scale, d.dtype = _row_stride(table, "table"), scale, dtype
    outp = _packed(out, table, "out", shape, table.dtype)
    if given:
        _written(out)
    _check(_lib.ms_embed(_on(d, table), tokens.data_ptr(), table.data_ptr(), outp))
    return out


def embed_grad(tokens, drows, vocab=None, scale=1.0, out=None, accumulate=False):
    """The gradient [vocab, dim] of `embed`'s table (ms_embed_grad): for each token, scale times the sum of its
    rows of drows [*tokens.shape, dim], in an order that depends on the tokens alone.

    float32, or the type of `out`; accumulate: added to what `out` holds."""
    dtype = _gpu(drows, range(1, 64), "drows [*tokens.shape, dim]")
    dim = drows.shape[-1]
    d = _embed_desc(tokens, drows)
    _like(drows, drows, "drows", (*tokens.shape, dim), drows.dtype)
    given = out is not None
    if not given:
        if accumulate or vocab is None:
            raise ValueError("accumulate needs out" if accumulate else "vocab or out is wanted")
        out = _torch.empty((vocab, dim), dtype=_torch.float32, device=drows.device)
    grad_dtype = _gpu(out, (2,), "out [vocab, dim]")
    _like(out, drows, "out", (out.shape[0] if vocab is None else vocab, dim), out.dtype)
    tokens, rows = tokens.contiguous(), drows.reshape(-1, dim)
    if (rows.shape[0] > 1 and rows.stride(0) < dim) or (dim > 1 and rows.stride(1) != 1):
        rows = rows.contiguous()   # a broadcast gradient, or columns apart
    d.vocab, d.dim = out.shape
    d.table_stride, d.row_stride = _row_stride(out, "out"), _row_stride(rows, "drows")
    d.scale, d.dtype, d.grad_dtype, d.accumulate = scale, dtype, grad_dtype, int(bool(accumulate))
    ref = _on(d, drows)
    hold, ws, n = _scratch(drows, _size(_lib.ms_embed_grad_workspace, ref))
    if given:
        _written(out)
    _check(_lib.ms_embed_grad(ref, tokens.data_ptr(), rows.data_ptr(), out.data_ptr(), ws, n))
    return out


# ----------------------------------------------------------------- gated lowpass
def _sequence(t, strides):
    """[batch, steps, dim] with contiguous channels, its strides written down; copied where they cannot be
    (two strides of 0 stand for a packed array)."""
    if t.is_contiguous():
        return t
    batch, steps, dim = t.shape
    sb, ss = t.stride(0) if batch > 1 else 0, t.stride(1) if steps > 1 else 0
    if (dim > 1 and t.stride(2) != 1) or sb == ss == 0:
        return t.contiguous()
    strides[0], strides[1] = sb, ss
    return t


def _gated_desc(v, g, y):
    dtype = _gpu(v, (3,), "v [batch, steps, dim]")
    _like(g, v, "g", v.shape, v.dtype)
    batch, steps, dim = v.shape
    d = GatedLowpassDesc(batch=batch, steps=steps, dim=dim, dtype=dtype)
    return d, _sequence(v, d.v_stride), _sequence(g, d.g_stride), y if y is None else _sequence(y, d.y_stride)


def gated_lowpass(v, g, y0=None, lengths=None, keep=False):
    """The lowpass synapse whose coefficient the input sets (ms_gated_lowpass): with a = sigmoid(g),
    y[:, t] = a[:, t] y[:, t-1] + (1 - a[:, t]) v[:, t] from y0 (zeros).

    v, g [batch, steps, dim], float32 or bfloat16; y0 [batch, dim] float32; lengths int32 [batch].
    Returns (y, last): y like v, zeros past a row's length, and the state after its last step, float32.
    keep: also the states that gated_lowpass_grad starts from."""
    d, v, g, _ = _gated_desc(v, g, None)
    batch, steps, dim = v.shape
    f32 = _torch.float32
    y = _torch.empty((batch, steps, dim), dtype=v.dtype, device=v.device)
    last = _torch.empty((batch, dim), dtype=f32, device=v.device)
    y0p, lp = _packed(y0, v, "y0", (batch, dim), f32), _packed(lengths, v, "lengths", (batch,), _torch.int32)
    ref = _on(d, v)
    kept = _torch.empty(_size(_lib.ms_gated_lowpass_kept, ref), dtype=f32, device=v.device) if keep else None
    hold, ws, n = _scratch(v, _size(_lib.ms_gated_lowpass_workspace, ref))
    _check(_lib.ms_gated_lowpass(ref, v.data_ptr(), g.data_ptr(), y0p, lp, y.data_ptr(), last.data_ptr(),
                                 kept.data_ptr() if keep else None, ws, n))
    return (y, last, kept) if keep else (y, last)


def gated_lowpass_grad(v, g, kept, dy, dlast=None, lengths=None):
    """(dv, dg, dy0) of gated_lowpass from dL/dy and dL/dlast (ms_gated_lowpass_grad); kept: what the forward
    call with keep=True left."""
    d, v, g, dy = _gated_desc(v, g, dy)
    _like(dy, v, "dy", v.shape, v.dtype)
    batch, steps, dim = v.shape
    f32 = _torch.float32
    dv = _torch.empty((batch, steps, dim), dtype=v.dtype, device=v.device)
    dg = _torch.empty((batch, steps, dim), dtype=v.dtype, device=v.device)
    dy0 = _torch.empty((batch, dim), dtype=f32, device=v.device)
    ref = _on(d, v)
    keptp = _packed(kept, v, "kept", (_size(_lib.ms_gated_lowpass_kept, ref),), f32)
    lp, dlp = _packed(lengths, v, "lengths", (batch,), _torch.int32), _packed(dlast, v, "dlast", (batch, dim), f32)
    hold, ws, n = _scratch(v, _size(_lib.ms_gated_lowpass_workspace, ref))
    _check(_lib.ms_gated_lowpass_grad(ref, v.data_ptr(), g.data_ptr(), keptp, lp, dy.data_ptr(), dlp, dv.data_ptr(),
                                      dg.data_ptr(), dy0.data_ptr(), ws, n))
    return dv, dg, dy0


def gated_lowpass_step(v, g, state, slots=None, out=None):
    """One step for the sequences being served (ms_gated_lowpass_step): row i of v, g [rows, dim] advances
    state[slots[i]] (float32 [slots, dim], in place; row i's own slot without `slots`, int32) and returns it in
    v's type; a slot outside the cache marks an idle row, whose result is zeros."""
    dtype = _gpu(v, (2,), "v [rows, dim]")
    rows, dim = shape = v.shape
    _like(g, v, "g", shape, v.dtype)
    _like(state, v, "state", (state.shape[0], dim), _torch.float32)
    written = (state,) if out is None else (state, out)
    if out is None:
        out = _torch.empty((rows, dim), dtype=v.dtype, device=v.device)
    else:
        _like(out, v, "out", shape, v.dtype)
    d = GatedStepDesc(rows, state.shape[0], dim, _row_stride(v, "v"), _row_stride(g, "g"), _row_stride(out, "out"),
                      _row_stride(state, "state"), dtype)
    slotp = _packed(slots, v, "slots", (rows,), _torch.int32)
    _written(*written)
    _check(_lib.ms_gated_lowpass_step(_on(d, v), v.data_ptr(), g.data_ptr(), state.data_ptr(), slotp, out.data_ptr()))
    return out


# ---------------------------------------------------------- orthogonalised updates
def _orth_desc(x, steps, coefficients, eps):
    dtype = _gpu(x, (2, 3), "a matrix or a batch of matrices")
    rows, cols = x.shape[-2:]
    batch = x.shape[0] if x.dim() == 3 else 1
    d = OrthDesc(batch=batch, rows=rows, cols=cols, eps=eps, steps=steps, dtype=dtype)
    d.coef[:] = coefficients
    if not x.is_contiguous():
        if (cols > 1 and x.stride(-1) != 1) or (rows > 1 and x.stride(-2) < cols):
            x = x.contiguous()
        else:
            d.x_stride[1] = x.stride(-2) if rows > 1 else cols
            d.x_stride[0] = x.stride(0) if x.dim() == 3 and batch > 1 else 0
    return d, x


def orthogonalise(x, steps=5, coefficients=NEWTON_SCHULZ, eps=1e-7, out=None):
    """Brings the singular values of a matrix [rows, cols], or of each of a batch, towards one
    (ms_orthogonalise): X <- (c0 I + c1 XX' + c2 XX'XX') X, `steps` times from X / (|X| + eps)."""
    d, x = _orth_desc(x, steps, coefficients, eps)
    given = out is not None
    if not given:
        out = _torch.empty(x.shape, dtype=x.dtype, device=x.device)
    outp = _packed(out, x, "out", x.shape, x.dtype)
    ref = _on(d, x)
    hold, ws, n = _scratch(x, _size(_lib.ms_orth_workspace, ref, 0))
    if given:
        _written(out)
    _check(_lib.ms_orthogonalise(ref, x.data_ptr(), outp, ws, n))
    return out


def orthogonal_update(weight, momentum, grad, rate, momentum_decay=0.95, weight_decay=0.0, nesterov=True, steps=5,
                      coefficients=NEWTON_SCHULZ, eps=1e-7):
    """One training step of a weight matrix, or a batch of them (ms_orthogonal_update), in place: momentum <-
    momentum_decay momentum + grad; weight <- (1 - rate weight_decay) weight - rate orthogonalise(grad +
    momentum_decay momentum), or of the momentum alone without nesterov.

    weight, momentum: float32, contiguous; grad: float32 or bfloat16."""
    d, grad = _orth_desc(grad, steps, coefficients, eps)
    f32 = _torch.float32
    wp, mp = _packed(weight, grad, "weight", grad.shape, f32), _packed(momentum, grad, "momentum", grad.shape, f32)
    rule = OrthRule(rate, momentum_decay, weight_decay, int(bool(nesterov)))
    ref = _on(d, grad)
    hold, ws, n = _scratch(grad, _size(_lib.ms_orth_workspace, ref, 1))
    _written(weight, momentum)
    _check(_lib.ms_orthogonal_update(ref, C.byref(rule), wp, mp, grad.data_ptr(), ws, n))
