"""Operators of an answer head on GPU tensors: layer norm, linear with its epilogue, log probabilities,
each with its gradient (include/ink.h has what they compute).

Argument marshalling only: every operator runs inside libink.so.  Calls are asynchronous on torch's
current stream of the tensors' device, like torch's own; results and work memory come from torch's
allocator.  Nothing is recorded for autograd: the gradients are calls of their own, and a tensor that requires a
gradient raises unless it is detached or the call stands under torch.no_grad().  A matrix is a 2-D
tensor whose rows are contiguous, at any distance from each other; any other layout is copied first.
Tensors of other devices or types and shapes that do not fit raise.
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


def _unrecorded(t, name):
    """Raises where autograd would expect a record of the call; t requires a gradient."""
    if torch.is_grad_enabled():
        raise ValueError("%s requires a gradient, and these operators record nothing for autograd: detach it or call under torch.no_grad(), "
                         "and use the *_backward calls" % name)


def _matrix(t, name, rows=None, cols=None, dtype=None, like=None):
    """t as a matrix of contiguous rows on a GPU, and the distance of its rows; raises where it is none or not of this
    shape, type and device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != 2:
        raise ValueError("%s must be a 2-D GPU tensor" % name)
    if t.dtype is not dtype and (dtype is not None or t.dtype not in TYPES):
        raise TypeError("%s has type %s, wanted %s" % (name, t.dtype, dtype or "float32, bfloat16 or float16"))
    n, m = t.shape
    if (rows is not None and n != rows) or (cols is not None and m != cols):
        raise ValueError("%s has shape %s, wanted [%s, %s]" % (name, tuple(t.shape), "rows" if rows is None else rows, m if cols is None else cols))
    if like is not None and t.device != like.device:
        raise ValueError("%s is on %s, the rows on %s" % (name, t.device, like.device))
    if t.requires_grad:
        _unrecorded(t, name)
    s0, s1 = t.stride()
    if (s1 != 1 and m > 1) or (s0 < m and s0 != 0 and n > 1):
        t = t.contiguous()
        s0 = m
    return t, s0


def _vector(t, name, n, like, dtypes):
    """t as a contiguous vector of n elements, or None as it is."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device != like.device or t.dim() != 1 or t.shape[0] != n:
        raise ValueError("%s must be a GPU tensor of shape [%d] on the rows' device" % (name, n))
    if t.dtype not in dtypes:
        raise TypeError("%s has type %s, wanted %s" % (name, t.dtype, " or ".join(str(d) for d in dtypes)))
    if t.requires_grad:
        _unrecorded(t, name)
    return t if n < 2 or t.stride(0) == 1 else t.contiguous()


def _given(t, name):
    """A tensor that this call cannot do without."""
    if t is None:
        raise ValueError("%s is missing" % name)
    return t


def _ptr(t):
    return None if t is None else t.data_ptr()


def _call(fn, like, *args):
    """fn(*args, stream) on the tensors' device; the raw-stream call is what torch's own stream objects are made from."""
    dev, had = like.device.index, torch._C._cuda_getDevice()
    if had == dev:
        status = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    if status != 0:
        raise InkError(status, _fn.ink_last_error(None).decode())


_F32 = (torch.float32,)


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd) of rows x: y = (x - mean) * rstd * weight + bias.  weight and bias: [cols] of x's type
    or float32 (both alike), or None; mean and rstd (float32) are what the gradient takes."""
    x, ld = _matrix(x, "x")
    rows, cols = x.shape
    t = x.dtype
    weight = _vector(weight, "weight", cols, x, (t, torch.float32))
    param = t if weight is None else weight.dtype
    bias = _vector(bias, "bias", cols, x, (t, torch.float32) if weight is None else (param,))
    if weight is None and bias is not None:
        param = bias.dtype
    lib = _functions()
    y = x.new_empty((rows, cols))
    mean, rstd = x.new_empty((2, rows), dtype=torch.float32).unbind(0)
    at = mean.data_ptr()
    _call(lib.ink_layer_norm, x, x.data_ptr(), ld, _ptr(weight), _ptr(bias), rows, cols, TYPES[t], TYPES[param], eps, y.data_ptr(), cols, at,
          at + 4 * rows)
    return y, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None, param_dtype=None, need_dx=True, need_params=True):
    """(dx, dweight, dbias) of layer_norm; None for what is not needed.  dweight and dbias have the weight's type,
    or param_dtype (x's type or float32) where there is no weight."""
    x, ld = _matrix(x, "x")
    rows, cols = x.shape
    t = x.dtype
    dy, ld_dy = _matrix(dy, "dy", rows, cols, t, x)
    mean, rstd = _vector(_given(mean, "mean"), "mean", rows, x, _F32), _vector(_given(rstd, "rstd"), "rstd", rows, x, _F32)
    weight = _vector(weight, "weight", cols, x, (t, torch.float32))
    if weight is not None:
        if param_dtype not in (None, weight.dtype):
            raise TypeError("param_dtype differs from the weight's type")
        param_dtype = weight.dtype
    elif param_dtype not in (None, t, torch.float32):
        raise TypeError("param_dtype must be x's type or float32")
    param_dtype = param_dtype or t
    lib = _functions()
    dx = x.new_empty((rows, cols)) if need_dx else None
    dweight = dbias = work = None
    n_work = 0
    if need_params:
        dweight, dbias = x.new_empty(cols, dtype=param_dtype), x.new_empty(cols, dtype=param_dtype)
        n_work = lib.ink_layer_norm_backward_work(rows, cols, TYPES[t])
        work = x.new_empty(n_work, dtype=torch.uint8) if n_work else None
    _call(lib.ink_layer_norm_backward, x, dy.data_ptr(), ld_dy, x.data_ptr(), ld, mean.data_ptr(), rstd.data_ptr(), _ptr(weight), rows, cols,
          TYPES[t], TYPES[param_dtype], _ptr(dx), cols, _ptr(dweight), _ptr(dbias), _ptr(work), n_work)
    return dx, dweight, dbias


def linear(x, weight, bias=None, act="none", residual=None, keep_pre=False, out_dtype=None):
    """act(x @ weight + bias) + residual, with weight [cols, out]; (y, z) with keep_pre, z = x @ weight + bias being what the
    gradient of an activation takes.  act: none, relu, gelu, silu.  out_dtype (type of y, z and residual): x's or float32."""
    x, ld = _matrix(x, "x")
    rows, cols = x.shape
    t = x.dtype
    weight, ld_w = _matrix(weight, "weight", cols, None, t, x)
    out = weight.shape[1]
    bias = _vector(bias, "bias", out, x, (t,))
    out_dtype = out_dtype or t
    if out_dtype is not t and out_dtype is not torch.float32:
        raise TypeError("out_dtype must be x's type or float32")
    if act not in ACTS:
        raise ValueError("act must be one of %s" % ", ".join(ACTS))
    ld_res = 0
    if residual is not None:
        residual, ld_res = _matrix(residual, "residual", rows, out, out_dtype, x)
    lib = _functions()
    y = x.new_empty((rows, out), dtype=out_dtype)
    pre = x.new_empty((rows, out), dtype=out_dtype) if keep_pre else None
    _call(lib.ink_linear, x, x.data_ptr(), ld, weight.data_ptr(), ld_w, _ptr(bias), _ptr(residual), ld_res, rows, cols, out, TYPES[t],
          TYPES[out_dtype], ACTS[act], y.data_ptr(), out, _ptr(pre), out)
    return (y, pre) if keep_pre else y


def linear_backward(dy, x, weight, pre=None, act="none", need_dx=True, need_dweight=True, need_dbias=True):
    """(dx, dweight, dbias) of linear, in the rows' type; None for what is not needed.  dy and pre (what linear kept, not
    needed for act "none") have x's type, or float32 with bfloat16 rows.  The gradient of the residual is dy."""
    x, ld = _matrix(x, "x")
    rows, cols = x.shape
    t = x.dtype
    weight, ld_w = _matrix(weight, "weight", cols, None, t, x)
    out = weight.shape[1]
    dy, ld_dy = _matrix(dy, "dy", rows, out, None, x)
    if dy.dtype is not t and not (dy.dtype is torch.float32 and t is torch.bfloat16):
        raise TypeError("dy has type %s, the rows %s: wanted the same, or float32 with bfloat16 rows" % (dy.dtype, t))
    if act not in ACTS:
        raise ValueError("act must be one of %s" % ", ".join(ACTS))
    ld_pre = 0
    if act == "none":
        pre = None
    else:
        pre, ld_pre = _matrix(pre, "pre", rows, out, dy.dtype, x)
    lib = _functions()
    dx = x.new_empty((rows, cols)) if need_dx else None
    dweight = x.new_empty((cols, out)) if need_dweight else None
    dbias = x.new_empty(out) if need_dbias else None
    n_work = lib.ink_linear_backward_work(rows, cols, out) if need_dweight or need_dbias else 0
    work = x.new_empty(n_work, dtype=torch.uint8) if n_work else None
    _call(lib.ink_linear_backward, x, dy.data_ptr(), ld_dy, x.data_ptr(), ld, weight.data_ptr(), ld_w, _ptr(pre), ld_pre, rows, cols, out,
          TYPES[t], TYPES[dy.dtype], ACTS[act], _ptr(dx), cols, _ptr(dweight), out, _ptr(dbias), _ptr(work), n_work)
    return dx, dweight, dbias


_INTEGERS = (torch.int64, torch.int32)


def log_probs(logits, targets=None, top=0, scale=1.0):
    """Of each row of logits, with p = softmax(scale * logits): dict of logp (log p of the row's target; 0 where the target is
    no class, -1 for instance), entropy, lse (all [rows] float32), and the `top` best classes: top_ids (int32) and
    top_logp, both [rows, top], best first and equal logits by the lower class."""
    logits, ld = _matrix(logits, "logits")
    rows, classes = logits.shape
    targets = _vector(targets, "targets", rows, logits, _INTEGERS)
    if not 0 <= top <= min(classes, MAX_TOP):
        raise ValueError("top must be 0 .. min(classes, %d)" % MAX_TOP)
    lib, t = _functions(), TYPES[logits.dtype]
    logp, entropy, lse = logits.new_empty((3, rows), dtype=torch.float32).unbind(0)
    ids = logits.new_empty((rows, top), dtype=torch.int32)
    top_logp = logits.new_empty((rows, top), dtype=torch.float32)
    n_work = lib.ink_log_probs_work(rows, classes, t, top)
    work = logits.new_empty(n_work, dtype=torch.uint8) if n_work else None
    at = logp.data_ptr()
    _call(lib.ink_log_probs, logits, logits.data_ptr(), ld, _ptr(targets), 0 if targets is None else targets.element_size(), rows, classes, t,
          scale, top, at, at + 4 * rows, at + 8 * rows, ids.data_ptr(), top_logp.data_ptr(), _ptr(work), n_work)
    return dict(logp=logp, entropy=entropy, lse=lse, top_ids=ids, top_logp=top_logp)


def log_probs_backward(logits, targets, lse, entropy=None, g_logp=None, g_entropy=None, scale=1.0):
    """Gradient by the logits of sum(g_logp * logp) + sum(g_entropy * entropy), in the logits' type.  lse and entropy are
    log_probs'; either gradient may be None (entropy is needed with g_entropy)."""
    logits, ld = _matrix(logits, "logits")
    rows, classes = logits.shape
    targets = _vector(targets, "targets", rows, logits, _INTEGERS)
    lse, entropy = _vector(_given(lse, "lse"), "lse", rows, logits, _F32), _vector(entropy, "entropy", rows, logits, _F32)
    g_logp, g_entropy = _vector(g_logp, "g_logp", rows, logits, _F32), _vector(g_entropy, "g_entropy", rows, logits, _F32)
    lib = _functions()
    out = logits.new_empty((rows, classes))
    _call(lib.ink_log_probs_backward, logits, logits.data_ptr(), ld, _ptr(targets), 0 if targets is None else targets.element_size(),
          lse.data_ptr(), _ptr(entropy), _ptr(g_logp), _ptr(g_entropy), rows, classes, TYPES[logits.dtype], scale, out.data_ptr(), classes)
    return out
