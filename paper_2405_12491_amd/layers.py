"""Layers that a student is trained with, on torch CUDA tensors.

``bridger_embed`` and ``bridger_embed_backward`` marshal device pointers to the C entry points of the
same names (include/bridger.h states formulas, types and limits).  ``embed`` and ``embed_grad`` follow
the rules of the row operators (operators.py): rows that are contiguous, at any distance, on any
device, launched on torch's current stream of that device, no CPU fallback.

A call whose inputs need a gradient is differentiated (once).  A stream that is being captured
refuses such calls: autograd keeps nodes on the streams they were made on, and a captured backward
pass that meets one of an eager graph ends the process.  There call the forward and the gradient's
function, ``embed_grad``, one after the other under ``torch.no_grad()``.
"""
from __future__ import annotations

import ctypes

import paper_2405_12491_amd as _B

from . import operators as _O
from .operators import _MOST, _call, _code, _ptr, _rows, _vector, _writable, _written

_P, _I32, _I64, _F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
_ARGTYPES = {
    "bridger_embed": [_P, _I64, _P, _P, _I64, _I32, _I64, _I32, _I32, _I32, _F, _P, _I64, _P],
    "bridger_embed_backward": [_P, _I64, _P, _P, _I64, _I32, _I64, _I32, _I32, _I32, _F, _P, _I64,
                               _P, _I64, _P],
}


def declare(lib):
    """Argument types of the layers' entry points."""
    for name, types in _ARGTYPES.items():
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = types, ctypes.c_int
    fn = lib.bridger_embed_backward_workspace
    fn.argtypes, fn.restype = [_I64, _I32, _I32, _I32], _I64


# ------------------------------------------------------------- raw entry points
def bridger_embed(ids_ptr, ldi, offsets_ptr, table_ptr, ldt, dtype, n_rows, n_slots, n_entries,
                  n_features, scale, out_ptr, ldo, stream=0):
    _B._check(_B.load_library().bridger_embed(
        ids_ptr, ldi, offsets_ptr, table_ptr, ldt, dtype, n_rows, n_slots, n_entries, n_features,
        scale, out_ptr, ldo, stream), "bridger_embed")


def bridger_embed_backward_workspace(n_rows, n_slots, n_entries, n_features) -> int:
    return _B.load_library().bridger_embed_backward_workspace(n_rows, n_slots, n_entries, n_features)


def bridger_embed_backward(ids_ptr, ldi, offsets_ptr, grad_ptr, ldg, dtype, n_rows, n_slots,
                           n_entries, n_features, scale, grad_table_ptr, ldt, workspace_ptr,
                           workspace_bytes, stream=0):
    _B._check(_B.load_library().bridger_embed_backward(
        ids_ptr, ldi, offsets_ptr, grad_ptr, ldg, dtype, n_rows, n_slots, n_entries, n_features,
        scale, grad_table_ptr, ldt, workspace_ptr, workspace_bytes, stream),
        "bridger_embed_backward")


# ------------------------------------------------------------------------- autograd
def _tracked(name, instead, *inputs):
    """Whether autograd has to see the call."""
    torch = _O._torch
    if not torch.is_grad_enabled():
        return False
    for t in inputs:
        if t is not None and getattr(t, "requires_grad", False):
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError(f"{name} with a gradient on a stream that is being captured: "
                                   f"take {instead}")
            return True
    return False


def _untracked_output(out, name):
    if out is not None:
        raise RuntimeError(f"{name} with a gradient does not write into outputs that are given")


_functions = {}


def _function(name, make):
    f = _functions.get(name)
    if f is None:
        f = _functions.setdefault(name, make(_O._torch))
    return f


def _once(torch, backward):
    """backward, which cannot be differentiated again, for a graph that may ask for that."""
    once = torch.autograd.function.once_differentiable(backward)

    def run(ctx, *grads):
        return (once if torch.is_grad_enabled() else backward)(ctx, *grads)
    return staticmethod(run)


# ---------------------------------------------------------------------------- embed
def _check_ids(ids, offsets, device):
    """(rows, slots, ids' and offsets' arguments)."""
    if getattr(ids, "dim", int)() == 1:
        ids = ids.unsqueeze(1)
    n, k, ldi = _rows(ids, "ids", None, None, _O._torch.int32, device)
    if offsets is not None:
        _vector(offsets, "offsets", k + 1, _O._torch.int64, ids.get_device())
    return n, k, (ids.data_ptr(), ldi, _ptr(offsets))


def _embed(ids, table, scale, offsets, out):
    n, k, first = _check_ids(ids, offsets, None)
    entries, w, ldt = _rows(table, "table", None, None, None, ids.get_device())
    code = _code(table.dtype)
    given = out
    if out is None:
        out, ldo = table.new_empty((n, w)), w
    else:
        ldo = _rows(out, "out", w, n, table.dtype, ids.get_device())[2]
        _writable(out, "out")
    _call("bridger_embed", table, *first, table.data_ptr(), ldt, code, n, k, entries, w, scale,
          out.data_ptr(), ldo)
    if given is not None:
        _written(given)
    return out


def _embed_grad(ids, grad, n_entries, scale, offsets, out):
    n, k, first = _check_ids(ids, offsets, None)
    _, w, ldg = _rows(grad, "grad", None, n, None, ids.get_device())
    code = _code(grad.dtype)
    if not 0 < n_entries <= _MOST:
        raise ValueError("n_entries must lie between 1 and 2^31 - 1")
    given = out
    if out is None:
        out, ldo = grad.new_empty((n_entries, w)), w
    else:
        ldo = _rows(out, "out", w, n_entries, grad.dtype, ids.get_device())[2]
        _writable(out, "out")
    bytes_ = _B._lib.bridger_embed_backward_workspace(n, k, n_entries, w)
    # (of at least one byte: an empty tensor has no address)
    workspace = grad.new_empty(max(bytes_, 1), dtype=_O._torch.uint8)
    _call("bridger_embed_backward", grad, *first, grad.data_ptr(), ldg, code, n, k, n_entries, w,
          scale, out.data_ptr(), ldo, workspace.data_ptr(), bytes_)
    if given is not None:
        _written(given)
    return out


def _make_embed(torch):
    class Embed(torch.autograd.Function):
        @staticmethod
        def forward(ctx, table, ids, offsets, scale):
            ctx.save_for_backward(ids, offsets)
            ctx.scale, ctx.entries = scale, table.shape[0]
            return _embed(ids, table, scale, offsets, None)

        def backward(ctx, grad):
            ids, offsets = ctx.saved_tensors
            return (_embed_grad(ids, grad.contiguous(), ctx.entries, ctx.scale, offsets, None),
                    None, None, None)
        backward = _once(torch, backward)
    return Embed


def embed(ids, table, scale: float = 1.0, offsets=None, out=None):
    """Rows of ``table`` [entries, width] that ``ids`` (int32 [n] or [n, slots]) name, added over a
    row's slots and times ``scale``: [n, width].  With ``offsets`` (int64 [slots + 1]) slot s reads
    the entries offsets[s] to offsets[s + 1] (a forest's leaves: predict_leaves' ids and the model's
    tree_offsets).  Ids outside are empty slots.  Differentiable in the table."""
    if _O._torch is None:
        _O._setup()
    if _tracked("embed", "embed and embed_grad under no_grad()", table):
        _untracked_output(out, "embed")
        return _function("embed", _make_embed).apply(table, ids, offsets, float(scale))
    return _embed(ids, table, float(scale), offsets, out)


def embed_grad(ids, grad, n_entries: int, scale: float = 1.0, offsets=None, out=None):
    """The gradient [n_entries, width] of embed's table, from that of its output ``grad``
    [n, width] (of its type).  The same ids give the same order of sums."""
    if _O._torch is None:
        _O._setup()
    return _embed_grad(ids, grad, int(n_entries), float(scale), offsets, out)
