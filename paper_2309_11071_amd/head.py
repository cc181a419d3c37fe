"""Operators of an answer head on GPU tensors: layer norm, linear with its epilogue, log probabilities,
each with its gradient (include/ink.h has what they compute).

Argument marshalling only: every operator runs inside libink.so.  Calls are asynchronous on torch's
current stream of the tensors' device, like torch's own; results and work memory come from torch's
allocator.  A matrix is a 2-D tensor whose rows are contiguous, at any distance from each other; any
other layout is copied first.  Tensors of other devices or types and shapes that do not fit raise.
"""
import ctypes as C

import torch

from .binding import InkError, load_library

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
MAX_TOP = 16

_fn = None


def _functions():
    global _fn
    if _fn is None:
        lib = load_library()
        p, i, l, f, z = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
        for name, args in dict(
                ink_layer_norm=(p, l, p, p, l, i, i, i, f, p, l, p, p, p),
                ink_layer_norm_backward=(p, l, p, l, p, p, p, l, i, i, i, p, l, p, p, p, z, p),
                ink_linear=(p, l, p, l, p, p, l, l, i, i, i, i, i, p, l, p, l, p),
                ink_linear_backward=(p, l, p, l, p, l, p, l, l, i, i, i, i, i, p, l, p, l, p, p, z, p),
                ink_log_probs=(p, l, p, i, l, l, i, f, i, p, p, p, p, p, p, z, p),
                ink_log_probs_backward=(p, l, p, i, p, p, p, p, l, l, i, f, p, l, p)).items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, C.c_int
        for name, args in dict(ink_layer_norm_backward_work=(l, i, i), ink_linear_backward_work=(l, i, i),
                               ink_log_probs_work=(l, l, i, i)).items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, z
        _fn = lib
    return _fn


def _check(lib, status):
    if status != 0:
        raise InkError(status, lib.ink_last_error(None).decode())


def _matrix(t, name, rows=None, cols=None, dtype=None, like=None):
    """t as a matrix of contiguous rows on a GPU; raises where it is none or not of this shape, type and device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != 2:
        raise ValueError("%s must be a 2-D GPU tensor" % name)
    if t.dtype not in TYPES or (dtype is not None and t.dtype != dtype):
        raise TypeError("%s has type %s, wanted %s" % (name, t.dtype, dtype or "float32, bfloat16 or float16"))
    n, m = t.shape
    if (rows is not None and n != rows) or (cols is not None and m != cols):
        raise ValueError("%s has shape %s, wanted [%s, %s]" % (name, tuple(t.shape), "rows" if rows is None else rows, m if cols is None else cols))
    if like is not None and t.device != like.device:
        raise ValueError("%s is on %s, the rows on %s" % (name, t.device, like.device))
    s0, s1 = t.stride()
    if (s1 != 1 and m > 1) or (s0 < m and s0 != 0 and n > 1):
        t = t.contiguous()
    return t


def _vector(t, name, n, like, dtypes):
    if not isinstance(t, torch.Tensor) or t.device != like.device or t.dim() != 1 or t.shape[0] != n:
        raise ValueError("%s must be a GPU tensor of shape [%d] on the rows' device" % (name, n))
    if t.dtype not in dtypes:
        raise TypeError("%s has type %s, wanted %s" % (name, t.dtype, " or ".join(str(d) for d in dtypes)))
    return t if t.is_contiguous() else t.contiguous()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(t):
    return torch.cuda.current_stream(t.device).cuda_stream


class _on:
    """Makes the tensors' device the current one for a call, where it is not."""

    def __init__(self, t):
        self.want = t.device.index

    def __enter__(self):
        self.had = torch.cuda.current_device()
        if self.had != self.want:
            torch.cuda.set_device(self.want)

    def __exit__(self, *_):
        if self.had != self.want:
            torch.cuda.set_device(self.had)


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd) of rows x: y = (x - mean) * rstd * weight + bias.  weight and bias: [cols] of x's type
    or float32 (both alike), or None; mean and rstd (float32) are what the gradient takes."""
    x = _matrix(x, "x")
    rows, cols = x.shape
    params = (x.dtype, torch.float32)
    weight = None if weight is None else _vector(weight, "weight", cols, x, params)
    bias = None if bias is None else _vector(bias, "bias", cols, x, params if weight is None else (weight.dtype,))
    param = weight if weight is not None else bias
    lib = _functions()
    y = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
    mean, rstd = (torch.empty(rows, dtype=torch.float32, device=x.device) for _ in range(2))
    with _on(x):
        _check(lib, lib.ink_layer_norm(x.data_ptr(), x.stride(0), _ptr(weight), _ptr(bias), rows, cols, TYPES[x.dtype],
                                       TYPES[x.dtype if param is None else param.dtype], eps, y.data_ptr(), cols, mean.data_ptr(),
                                       rstd.data_ptr(), _stream(x)))
    return y, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None, param_dtype=None, need_dx=True, need_params=True):
    """(dx, dweight, dbias) of layer_norm; None for what is not needed.  dweight and dbias have the weight's type,
    or param_dtype (x's type or float32) where there is no weight."""
    x = _matrix(x, "x")
    rows, cols = x.shape
    dy = _matrix(dy, "dy", rows, cols, x.dtype, x)
    mean, rstd = (_vector(v, n, rows, x, (torch.float32,)) for v, n in ((mean, "mean"), (rstd, "rstd")))
    if weight is not None:
        weight = _vector(weight, "weight", cols, x, (x.dtype, torch.float32))
        if param_dtype not in (None, weight.dtype):
            raise TypeError("param_dtype differs from the weight's type")
        param_dtype = weight.dtype
    elif param_dtype not in (None, x.dtype, torch.float32):
        raise TypeError("param_dtype must be x's type or float32")
    param_dtype = param_dtype or x.dtype
    lib = _functions()
    dx = torch.empty((rows, cols), dtype=x.dtype, device=x.device) if need_dx else None
    dweight = dbias = work = None
    n_work = 0
    if need_params:
        dweight, dbias = (torch.empty(cols, dtype=param_dtype, device=x.device) for _ in range(2))
        n_work = lib.ink_layer_norm_backward_work(rows, cols, TYPES[x.dtype])
        work = torch.empty(n_work, dtype=torch.uint8, device=x.device)
    with _on(x):
        _check(lib, lib.ink_layer_norm_backward(dy.data_ptr(), dy.stride(0), x.data_ptr(), x.stride(0), mean.data_ptr(), rstd.data_ptr(),
                                                _ptr(weight), rows, cols, TYPES[x.dtype], TYPES[param_dtype], _ptr(dx), cols,
                                                _ptr(dweight), _ptr(dbias), _ptr(work), n_work, _stream(x)))
    return dx, dweight, dbias


def linear(x, weight, bias=None, act="none", residual=None, keep_pre=False, out_dtype=None):
    """act(x @ weight + bias) + residual, with weight [cols, out]; (y, z) with keep_pre, z = x @ weight + bias being what the
    gradient of an activation takes.  act: none, relu, gelu, silu.  out_dtype (type of y, z and residual): x's or float32."""
    x = _matrix(x, "x")
    rows, cols = x.shape
    weight = _matrix(weight, "weight", cols, None, x.dtype, x)
    out = weight.shape[1]
    bias = None if bias is None else _vector(bias, "bias", out, x, (x.dtype,))
    out_dtype = out_dtype or x.dtype
    if out_dtype not in (x.dtype, torch.float32):
        raise TypeError("out_dtype must be x's type or float32")
    if act not in ACTS:
        raise ValueError("act must be one of %s" % ", ".join(ACTS))
    residual = None if residual is None else _matrix(residual, "residual", rows, out, out_dtype, x)
    lib = _functions()
    y = torch.empty((rows, out), dtype=out_dtype, device=x.device)
    pre = torch.empty_like(y) if keep_pre else None
    with _on(x):
        _check(lib, lib.ink_linear(x.data_ptr(), x.stride(0), weight.data_ptr(), weight.stride(0), _ptr(bias), _ptr(residual),
                                   0 if residual is None else residual.stride(0), rows, cols, out, TYPES[x.dtype], TYPES[out_dtype],
                                   ACTS[act], y.data_ptr(), out, _ptr(pre), out, _stream(x)))
    return (y, pre) if keep_pre else y


def linear_backward(dy, x, weight, pre=None, act="none", need_dx=True, need_dweight=True, need_dbias=True):
    """(dx, dweight, dbias) of linear, in the rows' type; None for what is not needed.  dy and pre (what linear kept, not
    needed for act "none") have x's type, or float32 with bfloat16 rows.  The gradient of the residual is dy."""
    x = _matrix(x, "x")
    rows, cols = x.shape
    weight = _matrix(weight, "weight", cols, None, x.dtype, x)
    out = weight.shape[1]
    dy = _matrix(dy, "dy", rows, out, None, x)
    if dy.dtype != x.dtype and not (dy.dtype == torch.float32 and x.dtype == torch.bfloat16):
        raise TypeError("dy has type %s, the rows %s: wanted the same, or float32 with bfloat16 rows" % (dy.dtype, x.dtype))
    if act not in ACTS:
        raise ValueError("act must be one of %s" % ", ".join(ACTS))
    if act == "none":
        pre = None
    else:
        pre = _matrix(pre, "pre", rows, out, dy.dtype, x)
    lib = _functions()
    dx = torch.empty((rows, cols), dtype=x.dtype, device=x.device) if need_dx else None
    dweight = torch.empty((cols, out), dtype=x.dtype, device=x.device) if need_dweight else None
    dbias = torch.empty(out, dtype=x.dtype, device=x.device) if need_dbias else None
    n_work = lib.ink_linear_backward_work(rows, cols, out) if need_dweight or need_dbias else 0
    work = torch.empty(n_work, dtype=torch.uint8, device=x.device) if n_work else None
    with _on(x):
        _check(lib, lib.ink_linear_backward(dy.data_ptr(), dy.stride(0), x.data_ptr(), x.stride(0), weight.data_ptr(), weight.stride(0),
                                            _ptr(pre), 0 if pre is None else pre.stride(0), rows, cols, out, TYPES[x.dtype],
                                            TYPES[dy.dtype], ACTS[act], _ptr(dx), cols, _ptr(dweight), out, _ptr(dbias), _ptr(work),
                                            n_work, _stream(x)))
    return dx, dweight, dbias


def _targets(t, rows, like):
    return None if t is None else _vector(t, "targets", rows, like, (torch.int64, torch.int32))


def log_probs(logits, targets=None, top=0, scale=1.0):
    """Of each row of logits, with p = softmax(scale * logits): dict of logp (log p of the row's target; 0 where the target is
    no class, -1 for instance), entropy, lse (all [rows] float32), and the `top` best classes: top_ids (int32) and
    top_logp, both [rows, top], best first and equal logits by the lower class."""
    logits = _matrix(logits, "logits")
    rows, classes = logits.shape
    targets = _targets(targets, rows, logits)
    if not 0 <= top <= min(classes, MAX_TOP):
        raise ValueError("top must be 0 .. min(classes, %d)" % MAX_TOP)
    lib, dev, t = _functions(), logits.device, TYPES[logits.dtype]
    logp, entropy, lse = (torch.empty(rows, dtype=torch.float32, device=dev) for _ in range(3))
    ids = torch.empty((rows, top), dtype=torch.int32, device=dev)
    top_logp = torch.empty((rows, top), dtype=torch.float32, device=dev)
    n_work = lib.ink_log_probs_work(rows, classes, t, top)
    work = torch.empty(n_work, dtype=torch.uint8, device=dev) if n_work else None
    with _on(logits):
        _check(lib, lib.ink_log_probs(logits.data_ptr(), logits.stride(0), _ptr(targets), 0 if targets is None else targets.element_size(),
                                      rows, classes, t, scale, top, logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(), ids.data_ptr(),
                                      top_logp.data_ptr(), _ptr(work), n_work, _stream(logits)))
    return dict(logp=logp, entropy=entropy, lse=lse, top_ids=ids, top_logp=top_logp)


def log_probs_backward(logits, targets, lse, entropy=None, g_logp=None, g_entropy=None, scale=1.0):
    """Gradient by the logits of sum(g_logp * logp) + sum(g_entropy * entropy), in the logits' type.  lse and entropy are
    log_probs'; either gradient may be None (entropy is needed with g_entropy)."""
    logits = _matrix(logits, "logits")
    rows, classes = logits.shape
    targets = _targets(targets, rows, logits)
    f32 = (torch.float32,)
    lse = _vector(lse, "lse", rows, logits, f32)
    entropy, g_logp, g_entropy = (None if v is None else _vector(v, n, rows, logits, f32)
                                  for v, n in ((entropy, "entropy"), (g_logp, "g_logp"), (g_entropy, "g_entropy")))
    lib = _functions()
    out = torch.empty((rows, classes), dtype=logits.dtype, device=logits.device)
    with _on(logits):
        _check(lib, lib.ink_log_probs_backward(logits.data_ptr(), logits.stride(0), _ptr(targets),
                                               0 if targets is None else targets.element_size(), lse.data_ptr(), _ptr(entropy),
                                               _ptr(g_logp), _ptr(g_entropy), rows, classes, TYPES[logits.dtype], scale, out.data_ptr(),
                                               classes, _stream(logits)))
    return out
