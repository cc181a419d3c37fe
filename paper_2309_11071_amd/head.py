"""Operators of an answer head on GPU tensors: layer norm, root-mean-square norm, linear with its epilogue, gated pairs of
projections, log probabilities, each with its gradient, and the step of AdamW that uses these (include/ink.h has what they compute).

Argument marshalling only: every operator runs inside libink.so.  Calls are asynchronous on torch's
current stream of the tensors' device, like torch's own; results and work memory come from torch's
allocator.  Nothing is recorded for autograd: the gradients are calls of their own, and a tensor that requires a
gradient raises unless it is detached or the call stands under torch.no_grad(); one with a tangent of forward mode raises unless it is detached.  A matrix is a 2-D
tensor whose rows are contiguous, at any distance from each other; any other layout is copied first.
Tensors of other devices or types and shapes that do not fit raise.
"""
import bisect
import ctypes as C
import itertools
import operator
import struct

import torch
from torch.autograd import forward_ad

from .binding import InkError, load_library

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
MAX_TOP = 16
E4M3 = torch.float8_e4m3fn
ADAMW_BLOCK = 128       # neighbouring elements whose 8-bit moments share a scale

_fn = None


def _functions():
    global _fn
    if _fn is None:
        lib = load_library()
        p, i, l, f, z, d, n = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t, C.c_double, C.c_uint64
        for name, args in dict(
                ink_layer_norm=(p, l, p, p, l, i, i, i, f, p, l, p, p, p),
                ink_layer_norm_backward=(p, l, p, l, p, p, p, l, i, i, i, p, l, p, p, p, z, p),
                ink_linear=(p, l, p, l, p, p, l, l, i, i, i, i, i, p, l, p, l, p),
                ink_linear_backward=(p, l, p, l, p, l, p, l, l, i, i, i, i, i, p, l, p, l, p, p, z, p),
                ink_log_probs=(p, l, p, i, l, l, i, f, i, p, p, p, p, p, p, z, p),
                ink_log_probs_backward=(p, l, p, i, p, p, p, p, l, l, i, f, p, l, p),
                ink_rms_norm=(p, l, p, l, p, l, i, i, i, f, i, p, l, p, p, l, p, p),
                ink_rms_norm_backward=(p, l, p, l, p, p, p, l, l, i, i, i, p, l, p, p, z, p),
                ink_gated=(p, l, p, p, l, p, l, p, p, l, i, i, i, i, i, p, l, p),
                ink_gated_backward=(p, l, p, l, p, l, p, l, l, i, i, i, i, p, l, p, l, p, l, p, z, p),
                ink_adamw=(p, i, i, i, i, i, d, d, d, d, d, l, p, d, p, n, p)).items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, C.c_int
        for name, args in dict(ink_layer_norm_backward_work=(l, i, i), ink_linear_backward_work=(l, i, i),
                               ink_log_probs_work=(l, l, i, i), ink_rms_norm_backward_work=(l, i, i),
                               ink_gated_backward_work=(l, i, i, i), ink_gated_backward_work_dx=(l, i, i)).items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, z
        _fn = lib
    return _fn


def _tangent(t, name):
    """Raises where forward mode would expect a tangent of the result (no_grad() does not concern it)."""
    if forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError("%s has a tangent, and these operators have no forward-mode derivatives: detach it" % name)


def _unrecorded(t, name):
    """Raises where autograd would expect a record of the call."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError("%s requires a gradient, and these operators record nothing for autograd: detach it or call under torch.no_grad(), "
                         "and use the *_backward calls" % name)
    _tangent(t, name)


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
    if t.requires_grad or forward_ad._current_level >= 0:
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
    if t.requires_grad or forward_ad._current_level >= 0:
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


def rms_norm(x, weight=None, residual=None, eps=1e-6, out_dtype=None):
    """(y, total, rstd) of rows x: total = x + residual in x's type (x itself without a residual), y = total * rstd * weight with
    rstd = 1 / sqrt(mean of total^2 + eps).  With out_dtype torch.float8_e4m3fn (y, scale, total, rstd): row r of the result is
    scale[r] times the numbers of y[r].  weight: [cols] of x's type or float32, or None; total and rstd are what the gradient takes."""
    x, ld = _matrix(x, "x")
    rows, cols = x.shape
    t = x.dtype
    weight = _vector(weight, "weight", cols, x, (t, torch.float32))
    out_dtype = out_dtype or t
    if out_dtype is not t and out_dtype is not E4M3:
        raise TypeError("out_dtype must be x's type or torch.float8_e4m3fn")
    total, ld_res, scale = x, 0, None
    if residual is not None:
        residual, ld_res = _matrix(residual, "residual", rows, cols, t, x)
        total = x.new_empty((rows, cols))
    lib = _functions()
    y = x.new_empty((rows, cols), dtype=out_dtype)
    rstd = x.new_empty(rows, dtype=torch.float32)
    if out_dtype is E4M3:
        scale = x.new_empty(rows, dtype=torch.float32)
    _call(lib.ink_rms_norm, x, x.data_ptr(), ld, _ptr(residual), ld_res, _ptr(weight), rows, cols, TYPES[t], TYPES[t if weight is None else weight.dtype],
          eps, _TYPES_8[out_dtype], y.data_ptr(), cols, _ptr(scale), None if residual is None else total.data_ptr(), cols, rstd.data_ptr())
    return (y, total, rstd) if scale is None else (y, scale, total, rstd)


def rms_norm_backward(dy, total, rstd, weight=None, d_total=None, param_dtype=None, need_dx=True, need_dweight=True):
    """(dx, dweight) of rms_norm; None for what is not needed.  dx is the gradient of x and of the residual alike, d_total (what arrives
    at the sum from elsewhere, or None) included.  dweight has the weight's type, or param_dtype (total's type or float32)
    where there is no weight."""
    total, ld = _matrix(total, "total")
    rows, cols = total.shape
    t = total.dtype
    dy, ld_dy = _matrix(dy, "dy", rows, cols, t, total)
    rstd = _vector(_given(rstd, "rstd"), "rstd", rows, total, _F32)
    weight = _vector(weight, "weight", cols, total, (t, torch.float32))
    ld_dt = 0
    if d_total is not None:
        d_total, ld_dt = _matrix(d_total, "d_total", rows, cols, t, total)
    if weight is not None:
        if param_dtype not in (None, weight.dtype):
            raise TypeError("param_dtype differs from the weight's type")
        param_dtype = weight.dtype
    elif param_dtype not in (None, t, torch.float32):
        raise TypeError("param_dtype must be total's type or float32")
    param_dtype = param_dtype or t
    lib = _functions()
    dx = total.new_empty((rows, cols)) if need_dx else None
    dweight = work = None
    n_work = 0
    if need_dweight:
        dweight = total.new_empty(cols, dtype=param_dtype)
        n_work = lib.ink_rms_norm_backward_work(rows, cols, TYPES[t])
        work = total.new_empty(n_work, dtype=torch.uint8) if n_work else None
    _call(lib.ink_rms_norm_backward, total, dy.data_ptr(), ld_dy, total.data_ptr(), ld, rstd.data_ptr(), _ptr(weight), _ptr(d_total), ld_dt, rows, cols,
          TYPES[t], TYPES[param_dtype], _ptr(dx), cols, _ptr(dweight), _ptr(work), n_work)
    return dx, dweight


_TYPES_8 = dict(TYPES)
_TYPES_8[E4M3] = 3


def _columns_8(w, name, cols, hidden, like):
    """8-bit weights [cols, hidden] as memory that holds a column's elements side by side, and the distance of its columns."""
    if not isinstance(w, torch.Tensor) or w.dim() != 2 or w.shape[0] != cols or (hidden is not None and w.shape[1] != hidden) or w.device != like.device:
        raise ValueError("%s must be a GPU tensor of shape [%d, %s] on the rows' device" % (name, cols, "hidden" if hidden is None else hidden))
    if w.dtype is not E4M3:
        raise TypeError("%s has type %s, wanted %s" % (name, w.dtype, E4M3))
    if w.requires_grad or forward_ad._current_level >= 0:
        _unrecorded(w, name)
    s0, s1 = w.stride()
    if (s0 != 1 and cols > 1) or (s1 < cols and s1 != 0 and w.shape[1] > 1):
        w = w.t().contiguous().t()
        s1 = cols
    return w, s1


def gated(x, w_gate, w_up, act="silu", x_scale=None, gate_scale=None, up_scale=None, out_dtype=None):
    """act(x @ w_gate) * (x @ w_up), with weights [cols, hidden] and act none, relu, gelu or silu, in x's type.

    Of 8-bit rows (torch.float8_e4m3fn, rms_norm's) with x_scale [rows] and 8-bit weights with gate_scale and up_scale [hidden] (all
    float32): rows and weights' columns are their numbers times their scales, and out_dtype is float32, bfloat16 (the default) or
    float16.  32-bit results have sums in 32 bits; for 16-bit ones, which take some 0.4 of the time, of every eight neighbouring products what lies below 2^-13 of
    the largest is dropped: less than the result's rounding but where large products cancel.  8-bit weights are taken as they are where a column's elements are side by side, as in the transpose of a
    contiguous [hidden, cols] tensor; any other layout is copied first."""
    if act not in ACTS:
        raise ValueError("act must be one of %s" % ", ".join(ACTS))
    scales = (x_scale, gate_scale, up_scale)
    if isinstance(x, torch.Tensor) and x.dtype is E4M3:
        x, ld = _matrix(x, "x", dtype=E4M3)
        rows, cols = x.shape
        w_gate, ld_gate = _columns_8(w_gate, "w_gate", cols, None, x)
        hidden = w_gate.shape[1]
        w_up, ld_up = _columns_8(w_up, "w_up", cols, hidden, x)
        x_scale, gate_scale, up_scale = (_vector(_given(v, name), name, n, x, _F32) for v, name, n in
                                         zip(scales, ("x_scale", "gate_scale", "up_scale"), (rows, hidden, hidden)))
        out_dtype = out_dtype or torch.bfloat16
        if out_dtype not in TYPES:
            raise TypeError("out_dtype must be float32, bfloat16 or float16")
    else:
        x, ld = _matrix(x, "x")
        rows, cols = x.shape
        if scales != (None, None, None):
            raise ValueError("scales go with 8-bit rows")
        w_gate, ld_gate = _matrix(w_gate, "w_gate", cols, None, x.dtype, x)
        hidden = w_gate.shape[1]
        w_up, ld_up = _matrix(w_up, "w_up", cols, hidden, x.dtype, x)
        if out_dtype not in (None, x.dtype):
            raise TypeError("out_dtype must be x's type")
        out_dtype = x.dtype
    lib = _functions()
    h = x.new_empty((rows, hidden), dtype=out_dtype)
    _call(lib.ink_gated, x, x.data_ptr(), ld, _ptr(x_scale), w_gate.data_ptr(), ld_gate, w_up.data_ptr(), ld_up, _ptr(gate_scale), _ptr(up_scale),
          rows, cols, hidden, _TYPES_8[x.dtype], TYPES[out_dtype], ACTS[act], h.data_ptr(), hidden)
    return h


def gated_backward(dh, x, w_gate, w_up, act="silu", need_dx=True, need_dweights=True):
    """(dx, dw_gate, dw_up) of gated, in x's type; None for what is not needed.  The projections are formed anew from x."""
    x, ld = _matrix(x, "x")
    rows, cols = x.shape
    t = x.dtype
    w_gate, ld_gate = _matrix(w_gate, "w_gate", cols, None, t, x)
    hidden = w_gate.shape[1]
    w_up, ld_up = _matrix(w_up, "w_up", cols, hidden, t, x)
    dh, ld_dh = _matrix(dh, "dh", rows, hidden, t, x)
    if act not in ACTS:
        raise ValueError("act must be one of %s" % ", ".join(ACTS))
    lib = _functions()
    dx = x.new_empty((rows, cols)) if need_dx else None
    dw_gate, dw_up = (x.new_empty((cols, hidden)), x.new_empty((cols, hidden))) if need_dweights else (None, None)
    n_work = 0
    if need_dweights:
        n_work = lib.ink_gated_backward_work(rows, cols, hidden, TYPES[t])
    elif need_dx:
        n_work = lib.ink_gated_backward_work_dx(rows, hidden, TYPES[t])
    work = x.new_empty(n_work, dtype=torch.uint8) if n_work else None
    _call(lib.ink_gated_backward, x, dh.data_ptr(), ld_dh, x.data_ptr(), ld, w_gate.data_ptr(), ld_gate, w_up.data_ptr(), ld_up, rows, cols, hidden,
          TYPES[t], ACTS[act], _ptr(dx), cols, _ptr(dw_gate), hidden, _ptr(dw_up), hidden, _ptr(work), n_work)
    return dx, dw_gate, dw_up


def adamw_moments(params, bits=32):
    """Moments of AdamW at the start, one entry for each parameter: (m, v) of 32 bits or (m, m_scale, v, v_scale) of 8."""
    if bits not in (8, 32):
        raise ValueError("moments have 32 or 8 bits")
    made = []
    for p in params:
        if bits == 32:
            made.append(tuple(torch.zeros(p.shape, dtype=torch.float32, device=p.device) for _ in range(2)))
        else:
            scales = torch.zeros((2, -(-p.numel() // ADAMW_BLOCK)), dtype=torch.float32, device=p.device)
            codes = [torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(E4M3) for _ in range(2)]
            made.append((codes[0], scales[0], codes[1], scales[1]))
    return made


_numel, _address, _contiguous, _device_index = torch.Tensor.numel, torch.Tensor.data_ptr, torch.Tensor.is_contiguous, torch.Tensor.get_device
_dtype, _shape, _requires_grad = operator.attrgetter("dtype"), operator.attrgetter("shape"), operator.attrgetter("requires_grad")


def _held(ts, name, sizes, dev, dtypes):
    """Addresses of the tensors that a step changes in place: contiguous, of these numbers of elements, on the GPU `dev`.  All of a list at
    a time: a head has hundreds of tensors, and a call should take less than the step."""
    types = set(map(_dtype, ts))
    if not types <= dtypes:
        raise TypeError("%s has type %s, wanted %s" % (name, (types - dtypes).pop(), " or ".join(sorted(map(str, dtypes)))))
    if set(map(_device_index, ts)) != {dev}:
        raise ValueError("%s is not on the parameters' GPU" % name)
    if list(map(_numel, ts)) != sizes:
        raise ValueError("%s has another number of elements than its parameter calls for" % name)
    if not all(map(_contiguous, ts)):
        raise ValueError("%s must be contiguous: the step changes it in place" % name)
    return list(map(_address, ts))


def _apart(changed, read):
    """Raises where extents (begin, end) in `changed` overlap each other, or one in `read` overlaps one of them."""
    begins, ends = sorted(b for b, _ in changed), sorted(e for _, e in changed)
    if any(map(operator.gt, ends, begins[1:])):                   # of disjoint extents every one ends before the next begins
        raise ValueError("tensors that the step changes overlap")
    if any(bisect.bisect_right(ends, b) != bisect.bisect_left(begins, e) for b, e in read):       # as many end before it as begin before its end
        raise ValueError("a gradient stands in the memory of a tensor that the step changes")


_PARAMS, _COPIES, _CODES, _SCALES = {torch.float32, torch.bfloat16}, {torch.bfloat16, torch.float16}, {E4M3}, {torch.float32}


def adamw(params, grads, moments, step, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_scale=1.0, copies=None, seed=0):
    """One step of AdamW over all of `params` (lists of tensors on one GPU, one entry for each), in place, in one launch for each 32 tensors.

    params: float32 or bfloat16, contiguous.  grads: float32, bfloat16 or float16, None where there is none (that parameter is left as it
    is).  moments: adamw_moments', all of one width.  copies: bfloat16 or float16 tensors that get the new float32 parameters (None, or a
    list with None where there is none).  step: the step's number, from 1, or an int64 GPU tensor of one element that holds it.
    grad_scale: a factor of every gradient, a number or a float32 GPU tensor of one element.  seed (64 bits): of the random numbers that round 8-bit
    moments and bfloat16 parameters up or down in proportion; they depend on seed, step, place in the list and element alone.  Roots of 8-bit second moments below 1/229376
    of their block's largest are held there."""
    n = len(params)
    if len(grads) != n or len(moments) != n or (copies is not None and len(copies) != n):
        raise ValueError("params, grads, moments and copies must have one entry for each parameter")
    place = [i for i in range(n) if grads[i] is not None]
    if not place:
        return
    some = len(place) < n
    p, g, mom = ([x[i] for i in place] for x in (params, grads, moments)) if some else (list(params), list(grads), moments)
    like, n = p[0], len(p)
    dev = like.get_device()
    if dev < 0:
        raise ValueError("params must be GPU tensors")
    width = len(mom[0])
    if width not in (2, 4) or set(map(len, mom)) != {width}:
        raise ValueError("moments must be adamw_moments', all of one width")
    sizes = list(map(_numel, p))
    at = _held(p, "a parameter", sizes, dev, _PARAMS)
    types = list(map(_dtype, p))
    if any(map(_requires_grad, p)) and torch.is_grad_enabled() and not all(x.is_leaf for x in p):
        raise ValueError("a parameter that requires a gradient and is no leaf cannot be changed in place")
    if not set(map(_dtype, g)) <= TYPES.keys() or set(map(_device_index, g)) != {dev} or list(map(_shape, g)) != list(map(_shape, p)):
        raise ValueError("a gradient must be a float32, bfloat16 or float16 tensor of its parameter's shape, on its GPU")
    if any(map(_requires_grad, g)) or forward_ad._current_level >= 0:
        for x in g:
            _unrecorded(x, "a gradient")
    if not all(map(_contiguous, g)):
        g = [x.contiguous() for x in g]
    if width == 2:
        held = [_held([m[0] for m in mom], "a first moment", sizes, dev, _SCALES), None, _held([m[1] for m in mom], "a second moment", sizes, dev, _SCALES), None]
    else:
        blocks = [-(-s // ADAMW_BLOCK) for s in sizes]
        held = [_held([m[0] for m in mom], "a first moment", sizes, dev, _CODES), _held([m[1] for m in mom], "a scale of first moments", blocks, dev, _SCALES),
                _held([m[2] for m in mom], "a second moment", sizes, dev, _CODES), _held([m[3] for m in mom], "a scale of second moments", blocks, dev, _SCALES)]
    none = [0] * n
    c, here, copy = none, [], none
    if copies is not None:
        copy = [copies[i] for i in place] if some else copies
        here = [i for i in range(n) if copy[i] is not None]
        if any(types[i] is not torch.float32 for i in here):
            raise TypeError("a copy is of float32 parameters")
        if here:
            c = list(none)
            for i, x in zip(here, _held([copy[i] for i in here], "a copy", [sizes[i] for i in here], dev, _COPIES)):
                c[i] = x
    if forward_ad._current_level >= 0:
        for x in itertools.chain(p, *mom, [copy[i] for i in here]):
            _tangent(x, "a tensor that the step changes")
    grad_at = list(map(_address, g))
    changed = [*at, *itertools.chain.from_iterable(h for h in held if h), *(x for x in c if x)]
    if not all(sizes):                                                        # tensors without elements have no address of their own
        changed = [x for column in (at, *held, c) if column for x, size in zip(column, sizes) if x and size]
    once = set(changed)
    if len(once) != len(changed):
        raise ValueError("a tensor that the step changes stands in the call twice")
    if not once.isdisjoint(grad_at if all(sizes) else [x for x, size in zip(grad_at, sizes) if size]):
        raise ValueError("a gradient stands in the memory of a tensor that the step changes")
    step_at = scale_at = None
    if isinstance(step, torch.Tensor):
        if step.dtype is not torch.int64 or step.numel() != 1 or step.get_device() != dev:
            raise ValueError("step must be a number or an int64 tensor of one element on the parameters' device")
        step_at, step = step.data_ptr(), 1
    if isinstance(grad_scale, torch.Tensor):
        if grad_scale.dtype is not torch.float32 or grad_scale.numel() != 1 or grad_scale.get_device() != dev:
            raise ValueError("grad_scale must be a number or a float32 tensor of one element on the parameters' device")
        if grad_scale.requires_grad or forward_ad._current_level >= 0:
            _unrecorded(grad_scale, "grad_scale")
        scale_at, grad_scale = grad_scale.data_ptr(), 1.0
    lib = _functions()
    columns = at, grad_at, c, held[0], held[2], held[1] or none, held[3] or none, sizes, place
    kinds = types, list(map(_dtype, g)), [None if x is None else x.dtype for x in copy] if here else none
    groups = {}
    if all(k.count(k[0]) == n for k in kinds):
        groups[tuple(k[0] for k in kinds)] = zip(*columns)
    else:
        for kind, entry in zip(zip(*kinds), zip(*columns)):
            groups.setdefault(kind, []).append(entry)
        extents = [[(x, x + s * w) for x, s, w in zip(column, sizes, widths) if x and s] for column, widths in
                   ((at, [x.element_size() for x in p]), (c, [2] * n), (held[0], [1 if width == 4 else 4] * n), (held[2], [1 if width == 4 else 4] * n))]
        extents += [[(x, x + 4 * b) for x, b in zip(held[i], blocks) if b] for i in (1, 3) if held[i]]
        read = [(x, x + s * y.element_size()) for x, s, y in zip(grad_at, sizes, g) if s]
        _apart(list(itertools.chain.from_iterable(extents)), read + [(x, x + b) for x, b in ((step_at, 8), (scale_at, 4)) if x])     # (a call finds its own overlaps)
    for (tp, tg, tc), entries in groups.items():
        numbers = list(itertools.chain.from_iterable(entries))
        table = struct.pack("%dq" % len(numbers), *numbers)
        _call(lib.ink_adamw, like, table, len(numbers) // len(columns), TYPES[tp], TYPES[tg], TYPES[tc] if tc else -1, 8 if width == 4 else 32, lr, betas[0],
              betas[1], eps, weight_decay, step, step_at, grad_scale, scale_at, seed & 0xFFFFFFFFFFFFFFFF)
    # what autograd has kept of these tensors is no longer what they hold
    torch.autograd.graph.increment_version(p)
    if here:
        torch.autograd.graph.increment_version([copy[i] for i in here])
