"""Operators over rows of scores, logits and features, on torch CUDA tensors.

``bridger_top_k``, ``bridger_distill``, ``bridger_distill_backward``, ``bridger_rmsnorm_q8`` and
``bridger_matmul_q8`` marshal device pointers to the C entry points of the same names
(include/bridger.h states formulas, types and limits).  ``top_k``, ``distill``, ``distill_loss``,
``rmsnorm_q8`` and ``matmul_q8`` take 2-D tensors whose rows are contiguous (any distance between
rows), on any device, and launch on torch's current stream of that device.  There is no CPU
fallback.
"""
from __future__ import annotations

import ctypes

import paper_2405_12491_amd as _B

BRIDGER_F32, BRIDGER_BF16, BRIDGER_F16 = 0, 1, 2
BRIDGER_MAX_TOP = 256
BRIDGER_MATMUL_Q8_MAX_FEATURES = 131071

_P, _I32, _I64, _F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
_ARGTYPES = {
    "bridger_top_k": [_P, _I64, _I32, _I64, _I32, _I32, _P, _P, _P],
    "bridger_distill": [_P, _I64, _I32, _P, _P, _I32, _I64, _I32, _I32, _F, _P, _P, _P, _P, _I64,
                        _P],
    "bridger_distill_backward": [_P, _I64, _I32, _P, _P, _I32, _I64, _I32, _I32, _F, _P, _P, _P,
                                 _I64, _P],
    "bridger_rmsnorm_q8": [_P, _I64, _P, _I64, _P, _I32, _I64, _I32, _F, _P, _I64, _P, _I64, _P,
                           _P],
    "bridger_matmul_q8": [_P, _I64, _P, _P, _I64, _P, _P, _I64, _I32, _I32, _I32, _P, _I64, _P],
}


def declare(lib):
    """Argument types of the operators' entry points."""
    for name, types in _ARGTYPES.items():
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = types, ctypes.c_int


# ------------------------------------------------------------- raw entry points
def bridger_top_k(scores_ptr, ld, dtype, n_rows, n_classes, k, values_ptr, ids_ptr, stream=0):
    _B._check(_B.load_library().bridger_top_k(scores_ptr, ld, dtype, n_rows, n_classes, k,
                                              values_ptr, ids_ptr, stream), "bridger_top_k")


def bridger_distill(logits_ptr, ldl, dtype, ids_ptr, teacher_ptr, teacher_dtype, n_rows, n_classes,
                    k, temperature, weight_ptr, loss_ptr, stats_ptr, grad_ptr, ldg, stream=0):
    _B._check(_B.load_library().bridger_distill(
        logits_ptr, ldl, dtype, ids_ptr, teacher_ptr, teacher_dtype, n_rows, n_classes, k,
        temperature, weight_ptr, loss_ptr, stats_ptr, grad_ptr, ldg, stream), "bridger_distill")


def bridger_distill_backward(logits_ptr, ldl, dtype, ids_ptr, teacher_ptr, teacher_dtype, n_rows,
                             n_classes, k, temperature, stats_ptr, weight_ptr, grad_ptr, ldg,
                             stream=0):
    _B._check(_B.load_library().bridger_distill_backward(
        logits_ptr, ldl, dtype, ids_ptr, teacher_ptr, teacher_dtype, n_rows, n_classes, k,
        temperature, stats_ptr, weight_ptr, grad_ptr, ldg, stream), "bridger_distill_backward")


def bridger_rmsnorm_q8(x_ptr, ldx, residual_ptr, ldr, weight_ptr, dtype, n_rows, n_features, eps,
                       total_ptr, ldt, q_ptr, ldq, scale_ptr, stream=0):
    _B._check(_B.load_library().bridger_rmsnorm_q8(
        x_ptr, ldx, residual_ptr, ldr, weight_ptr, dtype, n_rows, n_features, eps, total_ptr, ldt,
        q_ptr, ldq, scale_ptr, stream), "bridger_rmsnorm_q8")


def bridger_matmul_q8(a_ptr, lda, a_scale_ptr, b_ptr, ldb, b_scale_ptr, bias_ptr, n_rows, n_outputs,
                      n_features, dtype, out_ptr, ldo, stream=0):
    _B._check(_B.load_library().bridger_matmul_q8(
        a_ptr, lda, a_scale_ptr, b_ptr, ldb, b_scale_ptr, bias_ptr, n_rows, n_outputs, n_features,
        dtype, out_ptr, ldo, stream), "bridger_matmul_q8")


# ---------------------------------------------------------------- convenience
_codes = {}  # torch dtype -> BRIDGER_*


def _code(dtype) -> int:
    if not _codes:
        import torch
        _codes.update({torch.float32: BRIDGER_F32, torch.bfloat16: BRIDGER_BF16,
                       torch.float16: BRIDGER_F16})
    code = _codes.get(dtype)
    if code is None:
        raise TypeError(f"{dtype} rows: float32, bfloat16 or float16 are supported")
    return code


def _rows(t, name, width=None, n=None, dtype=None, device=None):
    """Checks a 2-D tensor with contiguous rows; the distance between its rows in elements."""
    import torch
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be of type {dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on another device")
    if t.dim() != 2 or (width is not None and t.shape[1] != width) or \
            (n is not None and t.shape[0] != n):
        raise ValueError(f"{name} must be [{'n' if n is None else n}, "
                         f"{'width' if width is None else width}]")
    w = t.shape[1]
    if w > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    if t.shape[0] <= 1:
        return w
    if t.stride(0) < w:
        raise ValueError(f"{name}'s rows overlap")
    return t.stride(0)


def _vector(t, name, n, dtype, device):
    import torch
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype):
        raise TypeError(f"{name} must be a {dtype} CUDA tensor")
    if t.device != device:
        raise ValueError(f"{name} is on another device")
    if t.dim() != 1 or t.shape[0] != n or not (n <= 1 or t.stride(0) == 1):
        raise ValueError(f"{name} must be contiguous [{n}]")


def _dense(t, name, n, width, dtype, device):
    if _rows(t, name, width, n, dtype, device) != width:
        raise ValueError(f"{name} must be contiguous")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _call(fn, device, *args):
    """Calls an entry point on the current stream of `device`, with that device current."""
    import torch
    stream = _B._launch_stream(device)
    if torch.cuda.current_device() == device.index:
        fn(*args, stream)
    else:
        with torch.cuda.device(device):
            fn(*args, stream)


def top_k(scores, k: int, values=None, ids=None):
    """The k largest of every row's scores, largest first (equal scores: the lower class first),
    and their class ids: (values [n, k] of scores' dtype, ids int32 [n, k]).  Slots beyond the
    number of classes hold -infinity and -1."""
    import torch
    ld = _rows(scores, "scores")
    n, c = scores.shape
    dev = scores.device
    if values is None:
        values = scores.new_empty((n, k))
    else:
        _dense(values, "values", n, k, scores.dtype, dev)
    if ids is None:
        ids = scores.new_empty((n, k), dtype=torch.int32)
    else:
        _dense(ids, "ids", n, k, torch.int32, dev)
    _call(bridger_top_k, dev, scores.data_ptr(), ld, _code(scores.dtype), n, c, k,
          values.data_ptr(), ids.data_ptr())
    return values, ids


def _check_distill(logits, ids, teacher, weight):
    import torch
    ld = _rows(logits, "logits")
    n, dev = logits.shape[0], logits.device
    if _rows(ids, "ids", None, n, torch.int32, dev) != ids.shape[1]:
        raise ValueError("ids must be contiguous")
    _dense(teacher, "teacher", n, ids.shape[1], teacher.dtype, dev)
    if weight is not None:
        _vector(weight, "weight", n, torch.float32, dev)
    return ld, _code(logits.dtype), _code(teacher.dtype)


def _forward(logits, ids, teacher, temperature, weight, loss, stats, grad):
    ld, code, teacher_code = _check_distill(logits, ids, teacher, weight)
    ldg = 0 if grad is None else _rows(grad, "grad", logits.shape[1], logits.shape[0],
                                       logits.dtype, logits.device)
    _call(bridger_distill, logits.device, logits.data_ptr(), ld, code, ids.data_ptr(),
          teacher.data_ptr(), teacher_code, logits.shape[0], logits.shape[1], ids.shape[1],
          float(temperature), _ptr(weight), _ptr(loss), _ptr(stats), _ptr(grad), ldg)


def distill(logits, ids, teacher, temperature: float = 1.0, weight=None, grad=None, loss=None):
    """Loss of every row [n] (float32) and its gradient [n, classes] (of logits' dtype), times
    ``weight`` [n] (float32), in one pass over the logits.  ``ids`` int32 and ``teacher`` [n, k]
    are the teacher's kept classes and their logits, as top_k gives them; ids outside the classes
    are empty slots.  ``grad`` may be ``logits`` itself."""
    import torch
    z = logits.detach() if isinstance(logits, torch.Tensor) else logits
    _rows(z, "logits")
    if loss is None:
        loss = z.new_empty((z.shape[0],), dtype=torch.float32)
    else:
        _vector(loss, "loss", z.shape[0], torch.float32, z.device)
    if grad is None:
        grad = torch.empty(z.shape, dtype=z.dtype, device=z.device)
    _forward(z, ids, teacher, temperature, weight, loss, None, grad)
    return loss, grad


_distill_function = None


def _make_distill_function():
    import torch

    class Distill(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, ids, teacher, temperature):
            loss = logits.new_empty((logits.shape[0],), dtype=torch.float32)
            stats = logits.new_empty((logits.shape[0], 2), dtype=torch.float32)
            _forward(logits, ids, teacher, temperature, None, loss, stats, None)
            ctx.save_for_backward(logits, ids, teacher, stats)
            ctx.temperature = temperature
            return loss

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad_loss):
            logits, ids, teacher, stats = ctx.saved_tensors
            weight = grad_loss.contiguous()
            grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
            ld, code, teacher_code = _check_distill(logits, ids, teacher, weight)
            _call(bridger_distill_backward, logits.device, logits.data_ptr(), ld, code,
                  ids.data_ptr(), teacher.data_ptr(), teacher_code, logits.shape[0],
                  logits.shape[1], ids.shape[1], ctx.temperature, stats.data_ptr(),
                  weight.data_ptr(), grad.data_ptr(), logits.shape[1])
            return grad, None, None, None

    return Distill


def distill_loss(logits, ids, teacher, temperature: float = 1.0):
    """distill's loss of every row [n], differentiable in ``logits`` (once; the teacher is taken
    as constant)."""
    global _distill_function
    if _distill_function is None:
        _distill_function = _make_distill_function()
    return _distill_function.apply(logits, ids, teacher, float(temperature))


def rmsnorm_q8(x, weight=None, residual=None, eps: float = 1e-6, q=None, scale=None, total=None):
    """Root-mean-square norm of every row of x (+ residual), times ``weight``, in 8 bits:
    (q int8 [n, f], scale float32 [n], total), q * scale[:, None] being the norm and total
    x + residual in x's dtype (None without a residual or a ``total`` to write).  ``total`` may be
    x or residual itself."""
    import torch
    ldx = _rows(x, "x")
    n, f = x.shape
    dev = x.device
    code = _code(x.dtype)
    ldr = 0 if residual is None else _rows(residual, "residual", f, n, x.dtype, dev)
    if weight is not None:
        _vector(weight, "weight", f, x.dtype, dev)
    if q is None:
        q = torch.empty((n, f), dtype=torch.int8, device=dev)
    if scale is None:
        scale = torch.empty((n,), dtype=torch.float32, device=dev)
    else:
        _vector(scale, "scale", n, torch.float32, dev)
    if total is None and residual is not None:
        total = torch.empty((n, f), dtype=x.dtype, device=dev)
    ldt = 0 if total is None else _rows(total, "total", f, n, x.dtype, dev)
    ldq = _rows(q, "q", f, n, torch.int8, dev)
    _call(bridger_rmsnorm_q8, dev, x.data_ptr(), ldx, _ptr(residual), ldr, _ptr(weight), code, n, f,
          float(eps), _ptr(total), ldt, q.data_ptr(), ldq, scale.data_ptr())
    return q, scale, total


def matmul_q8(a, a_scale, b, b_scale, bias=None, dtype=None, out=None):
    """a [n, f] times b [m, f] transposed, both int8 with float32 scales for each row of a [n] and
    of b [m], plus ``bias`` [m] (float32): [n, m] of ``dtype`` (bfloat16 unless given, or out's)."""
    import torch
    lda = _rows(a, "a", dtype=torch.int8)
    n, f = a.shape
    dev = a.device
    ldb = _rows(b, "b", f, None, torch.int8, dev)
    m = b.shape[0]
    _vector(a_scale, "a_scale", n, torch.float32, dev)
    _vector(b_scale, "b_scale", m, torch.float32, dev)
    if bias is not None:
        _vector(bias, "bias", m, torch.float32, dev)
    if out is None:
        out = torch.empty((n, m), dtype=dtype or torch.bfloat16, device=dev)
    ldo = _rows(out, "out", m, n, dtype, dev)
    _call(bridger_matmul_q8, dev, a.data_ptr(), lda, a_scale.data_ptr(), b.data_ptr(), ldb,
          b_scale.data_ptr(), _ptr(bias), n, m, f, _code(out.dtype), out.data_ptr(), ldo)
    return out
