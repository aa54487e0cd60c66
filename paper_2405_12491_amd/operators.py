"""Operators over rows of scores, logits and features, on torch CUDA tensors.

The functions named ``bridger_*`` marshal device pointers to the C entry points of the same names
(include/bridger.h states formulas, types and limits).  ``top_k``, ``sample``, ``distill``,
``distill_loss``, ``rmsnorm_q8`` and ``matmul_q8`` take 2-D tensors whose rows are contiguous (any distance between
rows), on any device, and launch on torch's current stream of that device.  There is no CPU
fallback.  Only ``distill_loss`` can be differentiated: the others pass no gradient and no tangent
on, whatever their inputs.  Outputs that the caller gives count as written in place: a backward pass
that still needs what was there raises, and one that requires grad is refused while gradients are
recorded.
"""
from __future__ import annotations

import ctypes

import paper_2405_12491_amd as _B

BRIDGER_F32, BRIDGER_BF16, BRIDGER_F16 = 0, 1, 2
BRIDGER_MAX_TOP = 256
BRIDGER_MATMUL_Q8_MAX_FEATURES = 131071
_MOST = 0x7FFFFFFF

_P, _I32, _I64, _F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
_D = ctypes.c_double
_ARGTYPES = {
    "bridger_top_k": [_P, _I64, _I32, _I64, _I32, _I32, _P, _P, _P],
    "bridger_sample": [_P, _I64, _I32, _I64, _I32, _P, _D, _P, _I32, _P, _D, _P, _D, _P, _P, _P, _P],
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


def bridger_sample(logits_ptr, ld, dtype, n_rows, n_classes, u_ptr, temperature, temperatures_ptr,
                   top_k, top_ks_ptr, top_p, top_ps_ptr, min_p, min_ps_ptr, ids_ptr, logp_ptr,
                   stream=0):
    _B._check(_B.load_library().bridger_sample(
        logits_ptr, ld, dtype, n_rows, n_classes, u_ptr, temperature, temperatures_ptr, top_k,
        top_ks_ptr, top_p, top_ps_ptr, min_p, min_ps_ptr, ids_ptr, logp_ptr, stream),
        "bridger_sample")


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
# A call on few rows is bound by its way to the launch: torch and its types are looked up once, a
# tensor's properties read once, and the entry points called without the functions above.
_torch = None
_forward_ad = None
_codes = {}  # torch dtype -> BRIDGER_*


def _setup():
    global _torch, _forward_ad
    import torch
    _forward_ad = torch.autograd.forward_ad
    _B.load_library()
    _codes.update({torch.float32: BRIDGER_F32, torch.bfloat16: BRIDGER_BF16,
                   torch.float16: BRIDGER_F16})
    _torch = torch  # last: other threads take it for the sign that all of this is done


def _code(dtype) -> int:
    code = _codes.get(dtype)
    if code is None:
        raise TypeError(f"{dtype} rows: float32, bfloat16 or float16 are supported")
    return code


def _rows(t, name, width, n, dtype, device):
    """Checks a 2-D tensor with contiguous rows (None: any): (rows, width, the distance between rows
    in elements)."""
    if not (isinstance(t, _torch.Tensor) and t.is_cuda):
        raise TypeError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be of type {dtype}")
    if device is not None and t.get_device() != device:
        raise ValueError(f"{name} is on another device")
    shape = t.shape
    if len(shape) != 2 or (width is not None and shape[1] != width) or \
            (n is not None and shape[0] != n):
        raise ValueError(f"{name} must be [{'n' if n is None else n}, "
                         f"{'width' if width is None else width}]")
    rows, w = shape
    if w > _MOST or rows > _MOST:  # more than the entry points' 32 bits hold
        raise ValueError(f"{name} has 2^31 or more rows or elements a row")
    step, inner = t.stride()
    if w > 1:
        if inner != 1:
            raise ValueError(f"{name}'s rows must be contiguous")
    elif t.is_neg():  # (such a view's elements are never neighbours)
        raise ValueError(f"{name} is a negated view: resolve_neg() it first")
    if rows <= 1:
        return rows, w, w
    if step < w:
        raise ValueError(f"{name}'s rows overlap")
    return rows, w, step


def _vector(t, name, n, dtype, device):
    if not (isinstance(t, _torch.Tensor) and t.is_cuda and t.dtype == dtype):
        raise TypeError(f"{name} must be a {dtype} CUDA tensor")
    if t.get_device() != device:
        raise ValueError(f"{name} is on another device")
    shape = t.shape
    if len(shape) != 1 or shape[0] != n or not (t.stride(0) == 1 if n > 1 else not t.is_neg()):
        raise ValueError(f"{name} must be contiguous [{n}]")


def _dense(t, name, n, width, dtype, device):
    if _rows(t, name, width, n, dtype, device)[2] != width:
        raise ValueError(f"{name} must be contiguous")


def _writable(t, name):
    """Refuses an output of the caller's whose gradient autograd would get wrong."""
    if t.requires_grad and _torch.is_grad_enabled():
        raise RuntimeError(f"{name} requires grad, and autograd does not see what is written into "
                           "it: give a detached tensor, or call under torch.no_grad()")


def _written(*outputs):
    """Tells autograd, which may keep them for a backward pass, that outputs of the caller's (None:
    none given) have been written."""
    for t in outputs:
        if t is not None:
            _torch.autograd.graph.increment_version(t)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _call(name, like, *args):
    """Calls an entry point on the current stream of `like`'s device, with that device current."""
    stream = _B._launch_stream(like.device)
    fn = getattr(_B._lib, name)
    if _torch.cuda.current_device() == like.get_device():
        st = fn(*args, stream)
    else:
        with _torch.cuda.device(like.device):
            st = fn(*args, stream)
    if st != _B.BRIDGER_OK:
        _B._check(st, name)


def top_k(scores, k: int, values=None, ids=None):
    """The k largest of every row's scores, largest first (equal scores: the lower class first),
    and their class ids: (values [n, k] of scores' dtype, ids int32 [n, k]).  Slots beyond the
    number of classes hold -infinity and -1."""
    if _torch is None:
        _setup()
    n, c, ld = _rows(scores, "scores", None, None, None, None)
    k, dev = int(k), scores.get_device()
    if not 1 <= k <= BRIDGER_MAX_TOP:
        raise ValueError("k must be between 1 and BRIDGER_MAX_TOP")
    given = None if values is None and ids is None else (values, ids)
    if values is None:
        values = scores.new_empty((n, k))
    else:
        _dense(values, "values", n, k, scores.dtype, dev)
        _writable(values, "values")
    if ids is None:
        ids = scores.new_empty((n, k), dtype=_torch.int32)
    else:
        _dense(ids, "ids", n, k, _torch.int32, dev)
    _call("bridger_top_k", scores, scores.data_ptr(), ld, _code(scores.dtype), n, c, k,
          values.data_ptr(), ids.data_ptr())
    if given:
        _written(*given)
    return values, ids


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, ids=None, logp=None):
    """A class of every row, drawn with the row's random number ``u`` (float32 [n], in [0, 1)) from
    the softmax of logits / temperature over the ``top_k`` largest (0: all) and, of those, the
    shortest leading part that holds ``top_p`` of their mass and the classes of at least ``min_p``
    times the largest probability: (ids int32 [n], logp float32 [n], the drawn class's logarithm of
    its share of what stays).  The four take a number, or a tensor [n] with a value for each row
    (float32, top_k int32).  A temperature of 0 takes the largest score.  A row of nothing but
    -infinity and NaN gives -1."""
    if _torch is None:
        _setup()
    n, c, ld = _rows(logits, "logits", None, None, None, None)
    dev, f32 = logits.get_device(), _torch.float32
    _vector(u, "u", n, f32, dev)
    given = ids is not None or logp is not None
    scalar, own = [], []
    for name, v, dtype, none in (("temperature", temperature, f32, 1.0),
                                 ("top_k", top_k, _torch.int32, 0), ("top_p", top_p, f32, 1.0),
                                 ("min_p", min_p, f32, 0.0)):
        if isinstance(v, _torch.Tensor):
            _vector(v, name, n, dtype, dev)
            scalar.append(none)
            own.append(v.data_ptr())
        else:
            scalar.append(type(none)(v))
            own.append(None)
    k = scalar[1]
    if not 0 <= k <= _MOST:
        raise ValueError("top_k must lie between 0 and 2^31 - 1")
    if ids is None:
        ids = logits.new_empty((n,), dtype=_torch.int32)
    else:
        _vector(ids, "ids", n, _torch.int32, dev)
    if logp is None:
        logp = u.new_empty((n,))
    else:
        _vector(logp, "logp", n, f32, dev)
        _writable(logp, "logp")
    _call("bridger_sample", logits, logits.data_ptr(), ld, _code(logits.dtype), n, c, u.data_ptr(),
          scalar[0], own[0], k, own[1], scalar[2], own[2], scalar[3], own[3], ids.data_ptr(),
          logp.data_ptr())
    if given:
        _written(ids, logp)
    return ids, logp


def _check_distill(logits, ids, teacher, weight):
    """What both passes take first, from checked tensors: (rows, classes, first arguments)."""
    n, c, ld = _rows(logits, "logits", None, None, None, None)
    dev = logits.get_device()
    _, k, step = _rows(ids, "ids", None, n, _torch.int32, dev)
    if step != k:
        raise ValueError("ids must be contiguous")
    _dense(teacher, "teacher", n, k, None, dev)
    if weight is not None:
        _vector(weight, "weight", n, _torch.float32, dev)
    return n, c, (logits.data_ptr(), ld, _code(logits.dtype), ids.data_ptr(), teacher.data_ptr(),
                  _code(teacher.dtype), n, c, k)


def distill(logits, ids, teacher, temperature: float = 1.0, weight=None, grad=None, loss=None):
    """Loss of every row [n] (float32) and its gradient [n, classes] (of logits' dtype), times
    ``weight`` [n] (float32), in one pass over the logits.  ``ids`` int32 and ``teacher`` [n, k]
    are the teacher's kept classes and their logits, as top_k gives them; ids outside the classes
    are empty slots.  ``grad`` may be ``logits`` itself.  Autograd does not see the call."""
    if _torch is None:
        _setup()
    n, c, args = _check_distill(logits, ids, teacher, weight)
    given = None if loss is None and grad is None else (loss, grad)
    if loss is None:
        loss = teacher.new_empty((n,), dtype=_torch.float32)
    else:
        _vector(loss, "loss", n, _torch.float32, logits.get_device())
        _writable(loss, "loss")
    if grad is None:
        grad, ldg = ids.new_empty((n, c), dtype=logits.dtype), c
    else:
        ldg = _rows(grad, "grad", c, n, logits.dtype, logits.get_device())[2]
        _writable(grad, "grad")
    _call("bridger_distill", logits, *args, float(temperature), _ptr(weight), loss.data_ptr(), None,
          grad.data_ptr(), ldg)
    if given:
        _written(*given)
    return loss, grad


_distill_function = None


def _make_distill_function():
    torch = _torch

    class Distill(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, ids, teacher, temperature):
            n, c, args = _check_distill(logits, ids, teacher, None)
            loss = ids.new_empty((n,), dtype=torch.float32)
            stats = ids.new_empty((n, 2), dtype=torch.float32)
            _call("bridger_distill", logits, *args, temperature, None, loss.data_ptr(),
                  stats.data_ptr(), None, 0)
            ctx.save_for_backward(logits, ids, teacher, stats)
            ctx.temperature, ctx.args, ctx.stride = temperature, args, logits.stride()
            return loss

        @staticmethod
        def backward(ctx, grad_loss):
            # with a graph of the backward pass: one that cannot be differentiated again
            return (once if torch.is_grad_enabled() else backward)(ctx, grad_loss)

    # Runs on autograd's own thread, where every step costs several times its usual time (10 us on
    # the caller's thread, 35 there): the forward pass's arguments serve again, unless hooks on
    # saved tensors gave other ones, and autograd has set the device.
    def backward(ctx, grad_loss):
        logits, ids, teacher, stats = ctx.saved_tensors
        args, weight = ctx.args, grad_loss.contiguous()
        if not (logits.data_ptr() == args[0] and logits.stride() == ctx.stride
                and ids.data_ptr() == args[3] and ids.is_contiguous()
                and teacher.data_ptr() == args[4] and teacher.is_contiguous()):
            args = _check_distill(logits, ids, teacher, weight)[2]
        grad = ids.new_empty(logits.shape, dtype=logits.dtype)
        st = _B._lib.bridger_distill_backward(
            *args, ctx.temperature, stats.data_ptr(), weight.data_ptr(), grad.data_ptr(), args[7],
            _B._launch_stream(grad.device))
        if st != _B.BRIDGER_OK:
            _B._check(st, "bridger_distill_backward")
        return grad, None, None, None

    once = torch.autograd.function.once_differentiable(backward)
    return Distill


def distill_loss(logits, ids, teacher, temperature: float = 1.0):
    """distill's loss of every row [n], differentiable in ``logits`` (once; the teacher is taken
    as constant).  Where logits need a gradient, a stream that is being captured is refused: autograd
    keeps nodes on the streams they were made on, and a captured backward pass that meets one of an
    eager graph ends the process.  (So the backward pass of a loss that was made outside does not
    belong into a capture either.)  There take distill and hand its gradient on
    (``logits.backward(grad)``)."""
    global _distill_function
    if _torch is None:
        _setup()
    if _distill_function is None:
        _distill_function = _make_distill_function()
    if getattr(logits, "requires_grad", False) and _torch.is_grad_enabled() and \
            _torch.cuda.is_current_stream_capturing():
        raise RuntimeError("distill_loss with a gradient on a stream that is being captured: "
                           "take distill")
    return _distill_function.apply(logits, ids, teacher, float(temperature))


def rmsnorm_q8(x, weight=None, residual=None, eps: float = 1e-6, q=None, scale=None, total=None):
    """Root-mean-square norm of every row of x (+ residual), times ``weight``, in 8 bits:
    (q int8 [n, f], scale float32 [n], total), q * scale[:, None] being the norm and total
    x + residual in x's dtype (None without a residual or a ``total`` to write).  ``total`` may be
    x or residual itself."""
    if _torch is None:
        _setup()
    n, f, ldx = _rows(x, "x", None, None, None, None)
    dev, dtype = x.get_device(), x.dtype
    code = _code(dtype)
    ldr = 0 if residual is None else _rows(residual, "residual", f, n, dtype, dev)[2]
    if weight is not None:
        _vector(weight, "weight", f, dtype, dev)
    given = None if q is None and scale is None and total is None else (q, scale, total)
    if q is None:
        q, ldq = x.new_empty((n, f), dtype=_torch.int8), f
    else:
        ldq = _rows(q, "q", f, n, _torch.int8, dev)[2]
    if scale is None:
        scale = x.new_empty((n,), dtype=_torch.float32)
    else:
        _vector(scale, "scale", n, _torch.float32, dev)
        _writable(scale, "scale")
    ldt = f
    if total is not None:
        ldt = _rows(total, "total", f, n, dtype, dev)[2]
        _writable(total, "total")
    elif residual is not None:
        total = x.new_empty((n, f))
    _call("bridger_rmsnorm_q8", x, x.data_ptr(), ldx, _ptr(residual), ldr, _ptr(weight), code, n, f,
          float(eps), _ptr(total), ldt, q.data_ptr(), ldq, scale.data_ptr())
    if given:
        _written(*given)
    return q, scale, total


def matmul_q8(a, a_scale, b, b_scale, bias=None, dtype=None, out=None):
    """a [n, f] times b [m, f] transposed, both int8 with float32 scales for each row of a [n] and
    of b [m], plus ``bias`` [m] (float32): [n, m] of ``dtype`` (bfloat16 unless given, or out's)."""
    if _torch is None:
        _setup()
    f32 = _torch.float32
    n, f, lda = _rows(a, "a", None, None, _torch.int8, None)
    dev = a.get_device()
    m, _, ldb = _rows(b, "b", f, None, _torch.int8, dev)
    _vector(a_scale, "a_scale", n, f32, dev)
    _vector(b_scale, "b_scale", m, f32, dev)
    if bias is not None:
        _vector(bias, "bias", m, f32, dev)
    given = out
    if out is None:
        dtype = dtype or _torch.bfloat16
        code = _code(dtype)
        out, ldo = a.new_empty((n, m), dtype=dtype), m
    else:
        ldo = _rows(out, "out", m, n, dtype, dev)[2]
        code = _code(out.dtype)
        _writable(out, "out")
    _call("bridger_matmul_q8", a, a.data_ptr(), lda, a_scale.data_ptr(), b.data_ptr(), ldb,
          b_scale.data_ptr(), _ptr(bias), n, m, f, code, out.data_ptr(), ldo)
    if given is not None:
        _written(given)
    return out
