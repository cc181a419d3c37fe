"""The operators of an answer head against their formulas in 64 bits, on the CPU.

Tolerances follow from the arithmetic: u = 2^-24 for 32-bit sums, U[type] for the final rounding; a sum whose longest chain of
additions is n terms errs by at most n u times the sum of the magnitudes, to first order.
"""
import math

import numpy as np
import pytest
import torch

from paper_2309_11071_amd import InkError, head

pytestmark = pytest.mark.gpu

u = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}       # spacing of subnormal numbers


def gen(seed):
    return torch.Generator().manual_seed(seed)


def table(x, ld=None, offset=0):
    """x on the GPU as rows `ld` apart that start `offset` elements into their memory."""
    rows, cols = x.shape
    ld = cols if ld is None else ld
    flat = torch.full((offset + max(rows, 1) * max(ld, 1) + 16,), float("nan"), dtype=x.dtype, device="cuda")
    v = flat[offset:].as_strided((rows, cols), (ld, 1))
    v.copy_(x)
    return v


def close(got, want, bound, dtype, what):
    """|got - want| <= bound + rounding of want to dtype; NaN and infinities in the same places."""
    got, want = got.double().cpu(), want.double()
    bound = torch.as_tensor(bound, dtype=torch.float64).expand_as(want)
    assert got.shape == want.shape, what
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    other = ~fine & ~torch.isnan(want)
    assert torch.equal(got[other], want[other]), what
    tol = bound + (want.abs() + bound) * U[dtype] + TINY[dtype]
    err = (got - want).abs()
    bad = fine & ~(err <= tol)
    assert not bad.any(), "%s: %d off, worst %.3g of its tolerance" % (what, int(bad.sum()), float((err / tol)[fine].max()))


# ------------------------------------------------------------------------------------ layer norm
CHAIN = 64          # a lane adds at most 32 elements, a group's sum takes at most 16 + 10 more


def norm_ref(x, w, b, eps):
    x = x.double()
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    rstd = (var + eps).rsqrt()
    h = (x - mean[:, None]) * rstd[:, None]
    e_mean = CHAIN * u * x.abs().mean(1) + u * mean.abs()
    # rstd: the centred squares' sum, with their error from the mean's
    e_rstd = rstd * (CHAIN * u + 8 * u + e_mean * rstd * 2)
    e_h = h.abs() * (e_rstd / rstd)[:, None] + rstd[:, None] * (e_mean[:, None] + 2 * u * (x.abs() + mean.abs()[:, None]))
    w = torch.ones(x.shape[1], dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(x.shape[1], dtype=torch.float64) if b is None else b.double()
    y = h * w + b
    return y, mean, rstd, e_h * w.abs() + 4 * u * ((h * w).abs() + b.abs()), e_mean, e_rstd


NORM_SHAPES = [(1, 1), (3, 2), (2, 3), (1, 7), (5, 8), (1, 9), (33, 16), (2, 41), (65, 47), (7, 64), (130, 100), (1, 128), (257, 128), (9, 172),
               (64, 256), (31, 257), (3, 512), (17, 602), (5, 1000), (3, 1024), (2, 2047), (2, 2049), (1, 4100), (2, 8192), (1, 16384), (3, 16383)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
def test_layer_norm(rows, cols, dtype):
    g = gen(rows * 31 + cols)
    x = (torch.randn(rows, cols, generator=g) * 2 + 1).to(dtype)
    w, b = (1 + 0.3 * torch.randn(cols, generator=g)).to(dtype), torch.randn(cols, generator=g).to(dtype)
    for ld, off, pw, pb in ((cols, 0, w, b), (cols + 3, 1, w.float(), None), (cols + 16, 0, None, b), (2 * cols + 1, 3, None, None)):
        y, mean, rstd = head.layer_norm(table(x, ld, off), None if pw is None else pw.cuda(), None if pb is None else pb.cuda(), eps=1e-5)
        want = norm_ref(x, pw, pb, 1e-5)
        close(y, want[0], want[3], dtype, "y")
        close(mean, want[1], want[4], F32, "mean")
        close(rstd, want[2], want[5], F32, "rstd")


def norm_grad_ref(dy, x, mean, rstd, w):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    w = torch.ones(x.shape[1], dtype=torch.float64) if w is None else w.double()
    h = (x - mean) * rstd
    g = dy * w
    dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    e_h = 3 * u * rstd * (x.abs() + mean.abs())
    a_g, a_gh = g.abs().mean(1, keepdim=True), (g * h).abs().mean(1, keepdim=True)
    e = rstd.abs() * (8 * u * (g.abs() + a_g + h.abs() * a_gh) + CHAIN * u * (a_g + h.abs() * a_gh)
                      + e_h * a_gh + h.abs() * (g.abs() * e_h).mean(1, keepdim=True))
    n = len(x) + 64
    return (dx, (dy * h).sum(0), dy.sum(0), e, n * u * (dy * h).abs().sum(0) + (dy.abs() * e_h).sum(0), n * u * dy.abs().sum(0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", NORM_SHAPES + [(5000, 47), (3001, 256), (2100, 602), (700, 2050)])
def test_layer_norm_backward(rows, cols, dtype):
    g = gen(rows * 17 + cols)
    x, dy = ((torch.randn(rows, cols, generator=g) * 2 + 1).to(dtype) for _ in range(2))
    w = (1 + 0.3 * torch.randn(cols, generator=g)).to(dtype)
    _, mean, rstd, *_ = norm_ref(x, None, None, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    for ld, off, pw in ((cols, 0, w), (cols + 5, 1, w.float()), (cols + 2, 2, None)):
        dx, dw, db = head.layer_norm_backward(table(dy, ld, off), table(x, ld + 1, off), mean.cuda(), rstd.cuda(), None if pw is None else pw.cuda())
        want = norm_grad_ref(dy, x, mean, rstd, pw)
        p = dtype if pw is None else pw.dtype
        assert dw.dtype == db.dtype == p
        close(dx, want[0], want[3], dtype, "dx")
        close(dw, want[1], want[4], p, "dweight")
        close(db, want[2], want[5], p, "dbias")
    dx2, none, none2 = head.layer_norm_backward(dy.cuda(), x.cuda(), mean.cuda(), rstd.cuda(), need_params=False)
    assert none is None and none2 is None and torch.equal(dx2, head.layer_norm_backward(dy.cuda(), x.cuda(), mean.cuda(), rstd.cuda())[0])
    none, dw, db = head.layer_norm_backward(dy.cuda(), x.cuda(), mean.cuda(), rstd.cuda(), need_dx=False, param_dtype=F32)
    want = norm_grad_ref(dy, x, mean, rstd, None)
    assert none is None
    close(dw, want[1], want[4], F32, "dweight alone")
    close(db, want[2], want[5], F32, "dbias alone")


def test_layer_norm_gradient_against_differences():
    """The kernels' gradient against central differences of the formula in 64 bits (step 1e-5: truncation and rounding below 1e-8)."""
    g = gen(3)
    x, dy = torch.randn(3, 11, generator=g), torch.randn(3, 11, generator=g)
    w, b = torch.randn(11, generator=g), torch.randn(11, generator=g)
    _, mean, rstd = head.layer_norm(x.cuda(), w.cuda(), b.cuda())
    dx, dw, db = head.layer_norm_backward(dy.cuda(), x.cuda(), mean, rstd, w.cuda())

    def loss(x_, w_, b_):
        return float((norm_ref(x_, w_, b_, 1e-5)[0] * dy.double()).sum())
    differences(loss, [x, w, b], [dx, dw, db], 2e-5)


def differences(loss, at, grads, tol):
    at = [t.double() for t in at]
    for k, t in enumerate(at):
        for i in range(t.numel()):
            lo, hi = t.clone(), t.clone()
            lo.view(-1)[i] -= 1e-5
            hi.view(-1)[i] += 1e-5
            d = (loss(*at[:k], hi, *at[k + 1:]) - loss(*at[:k], lo, *at[k + 1:])) / 2e-5
            got = float(grads[k].reshape(-1)[i])
            assert abs(got - d) <= tol * max(1.0, abs(d)), (k, i, got, d)


def test_layer_norm_constant_and_special_rows():
    x = torch.zeros(6, 100)
    x[1] = 7.25
    x[2, 5] = float("nan")
    x[3, 5] = float("inf")
    x[4] = torch.arange(100) * 3e16        # the squares' sum, 7.5e37, is within the range of 32 bits
    x[5, ::2] = 1e-20                      # variance below eps
    y, mean, rstd = head.layer_norm(x.cuda(), eps=1e-5)
    y = y.cpu()
    assert torch.equal(y[0], torch.zeros(100)) and torch.equal(y[1], torch.zeros(100))
    assert math.isclose(float(rstd[1]), 1e-5 ** -0.5, rel_tol=1e-6)
    assert torch.isnan(y[2]).all() and torch.isnan(y[3]).all()
    assert torch.isfinite(y[4]).all() and abs(float(y[4].mean())) < 1e-5
    assert torch.isfinite(y[5]).all()


# ------------------------------------------------------------------------------------ linear
def act_ref(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def act_grad_ref(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def linear_case(rows, cols, out, dtype, seed):
    g = gen(seed)
    x = torch.randn(rows, cols, generator=g).to(dtype)
    w = (torch.randn(cols, out, generator=g) / math.sqrt(cols)).to(dtype)
    return g, x, w, torch.randn(out, generator=g).to(dtype)


def linear_ref(x, w, b, act, res):
    z = x.double() @ w.double()
    mag = x.double().abs() @ w.double().abs()
    if b is not None:
        z, mag = z + b.double(), mag + b.double().abs()
    e_z = (x.shape[1] + 4) * u * mag
    y = act_ref(z, act)
    e_y = 1.13 * e_z + (2e-7 * z.abs() + 8 * u * y.abs() if act in ("gelu", "silu") else 0)   # 1.13: the steepest slope
    if res is not None:
        y, e_y = y + res.double(), e_y + 2 * u * (y.abs() + res.double().abs())
    return y, z, e_y, e_z


LINEAR_SHAPES = [(1, 1, 1), (1, 602, 256), (3, 5, 7), (16, 128, 47), (17, 128, 47), (2, 16, 172), (33, 15, 33), (40, 64, 64), (100, 100, 41),
                 (129, 256, 100), (300, 602, 256), (257, 33, 300), (513, 128, 172), (70, 1000, 513), (1000, 7, 8), (260, 2050, 65)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,out", LINEAR_SHAPES)
def test_linear(rows, cols, out, dtype):
    g, x, w, b = linear_case(rows, cols, out, dtype, rows + cols + out)
    r = torch.randn(rows, out, generator=g)
    for act, res, bias, f32, pad in (("none", False, True, False, 0), ("gelu", True, True, False, 1), ("relu", True, False, True, 8), ("silu", False, True, True, 3)):
        to = F32 if f32 else dtype
        rr = r.to(to) if res else None
        y, z = head.linear(table(x, cols + pad, pad), table(w, out + pad, pad), b.cuda() if bias else None, act=act,
                           residual=None if rr is None else table(rr, out + pad, pad), keep_pre=True, out_dtype=to)
        want = linear_ref(x, w, b if bias else None, act, rr)
        assert y.dtype == z.dtype == to
        close(z, want[1], want[3], to, "z " + act)
        close(y, want[0], want[2], to, "y " + act)
        y2 = head.linear(x.cuda(), w.cuda(), b.cuda() if bias else None, act=act, residual=None if rr is None else rr.cuda(), out_dtype=to)
        assert torch.equal(y, y2), "the layout of the tensors changed the result"


# enough rows for the kernels that keep W in registers, or for their fallback (deep sums): every class of depth and width, sizes beside
# the tiles', a last tile of one row
MANY = [(32769, 128, 47), (33000, 100, 64), (32800, 128, 128), (32769, 64, 172), (32768, 200, 41), (32790, 256, 256), (32769, 255, 100), (32801, 300, 47),
        (32769, 602, 128), (33001, 602, 256), (32769, 640, 300), (32769, 7, 9), (33333, 3, 5), (32769, 650, 70), (32777, 33, 1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,out", MANY)
def test_linear_many_rows(rows, cols, out, dtype):
    g, x, w, b = linear_case(rows, cols, out, dtype, rows + 7 * cols + out)
    r = torch.randn(rows, out, generator=g)
    for act, res, bias, f32, pad in (("gelu", True, True, False, 0), ("relu", True, False, True, 5), ("silu", False, True, False, 2)):
        to = F32 if f32 else dtype
        rr = r.to(to) if res else None
        args = (b.cuda() if bias else None, act, None if rr is None else table(rr, out + pad, pad))
        y, z = head.linear(table(x, cols + pad, pad), table(w, out + pad, pad), *args, keep_pre=True, out_dtype=to)
        want = linear_ref(x, w, b if bias else None, act, rr)
        close(z, want[1], want[3], to, "z " + act)
        close(y, want[0], want[2], to, "y " + act)
        assert torch.equal(y, head.linear(x.cuda(), w.cuda(), *args, out_dtype=to))
    view = torch.full((rows, out + 9), 7.0, dtype=dtype, device="cuda")       # results as columns of a wider table: nothing beside them is written
    wide = table(x)
    lib, stream = head._functions(), torch.cuda.current_stream().cuda_stream
    wd = w.cuda()
    assert lib.ink_linear(wide.data_ptr(), cols, wd.data_ptr(), out, None, None, 0, rows, cols, out, head.TYPES[dtype], head.TYPES[dtype], 0,
                          view[:, 4:].data_ptr(), out + 9, None, 0, stream) == 0
    torch.cuda.synchronize()
    want = linear_ref(x, w, None, "none", None)
    close(view[:, 4:4 + out], want[0], want[2], dtype, "columns of a table")
    assert (view[:, :4] == 7).all() and (view[:, 4 + out:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,out", MANY)
def test_linear_backward_many_rows(rows, cols, out, dtype):
    g, x, w, _ = linear_case(rows, cols, out, dtype, rows * 5 + cols + out)
    dy, pre = torch.randn(rows, out, generator=g), 2 * torch.randn(rows, out, generator=g)
    for act, f32, pad in (("none", False, 1), ("gelu", True, 0), ("silu", False, 4)):
        to = F32 if f32 and dtype == BF16 else dtype
        d, p = dy.to(to), pre.to(to)
        got = head.linear_backward(table(d, out + pad, pad), table(x, cols + pad, pad), table(w, out + pad, pad),
                                   pre=None if act == "none" else table(p, out + 2 * pad, pad), act=act)
        want = linear_grad_ref(d, x, w, p, act, dtype)
        for i, name in enumerate(("dx", "dweight", "dbias")):
            close(got[i], want[i], want[3 + i], dtype, name + " " + act)


def linear_grad_ref(dy, x, w, pre, act, dtype):
    dz = dy.double()
    e = torch.zeros_like(dz)
    if act != "none":
        z = pre.double()
        e = dz.abs() * (1e-6 + 8 * u) * (1 + z.abs())        # the distribution function's 1.5e-7 and the density's rounding, with room
        dz = dz * act_grad_ref(z, act)
    e_r = e + (0 if dtype == F32 else U[dtype] * dz.abs() + TINY[dtype])      # rounded before the products
    aw, ax = w.double().abs(), x.double().abs()
    n, k = dz.shape[1] + 4, len(x) + 600
    return (dz @ w.double().T, x.double().T @ dz, dz.sum(0),
            e_r @ aw.T + n * u * dz.abs() @ aw.T, ax.T @ e_r + k * u * ax.T @ dz.abs(), e.sum(0) + k * u * dz.abs().sum(0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,out", LINEAR_SHAPES + [(5000, 128, 47), (3000, 100, 172), (2500, 256, 256)])
def test_linear_backward(rows, cols, out, dtype):
    g, x, w, _ = linear_case(rows, cols, out, dtype, rows * 3 + cols + out)
    dy, pre = torch.randn(rows, out, generator=g), 2 * torch.randn(rows, out, generator=g)
    for act, f32, pad in (("none", False, 0), ("gelu", False, 1), ("relu", True, 8), ("silu", True, 3)):
        to = F32 if f32 and dtype == BF16 else dtype
        d, p = dy.to(to), pre.to(to)
        got = head.linear_backward(table(d, out + pad, pad), table(x, cols + pad, pad), table(w, out + pad, pad),
                                   pre=None if act == "none" else table(p, out + 2 * pad, pad), act=act)
        want = linear_grad_ref(d, x, w, p, act, dtype)
        for i, name in enumerate(("dx", "dweight", "dbias")):
            assert got[i].dtype == dtype
            close(got[i], want[i], want[3 + i], dtype, name + " " + act)
        parts = [head.linear_backward(d.cuda(), x.cuda(), w.cuda(), pre=p.cuda(), act=act, need_dx=i == 0, need_dweight=i == 1, need_dbias=i == 2)
                 for i in range(3)]
        for i in range(3):
            assert [v is None for v in parts[i]] == [j != i for j in range(3)]
            close(parts[i][i], want[i], want[3 + i], dtype, "one gradient alone")


@pytest.mark.parametrize("act", ["gelu", "silu", "none"])
def test_linear_gradient_against_differences(act):
    g = gen(5)
    x, w, b, dy = torch.randn(3, 6, generator=g), torch.randn(6, 5, generator=g), torch.randn(5, generator=g), torch.randn(3, 5, generator=g)
    _, z = head.linear(x.cuda(), w.cuda(), b.cuda(), act=act, keep_pre=True)
    grads = head.linear_backward(dy.cuda(), x.cuda(), w.cuda(), pre=z, act=act)

    def loss(x_, w_, b_):
        return float((act_ref(x_ @ w_ + b_, act) * dy.double()).sum())
    differences(loss, [x, w, b], grads, 2e-5)


def test_linear_special_values():
    """NaN and infinity stay in their rows; what lies beside a matrix in memory is not read into it."""
    x = torch.randn(40, 37, generator=gen(1))
    x[3, 36], x[5, 0], x[39, 1] = float("nan"), float("inf"), 1e30
    w = torch.ones(37, 9)
    for dtype in TYPES:
        if dtype == F16:
            x[39, 1] = 6e4
        for act in ("none", "relu", "gelu", "silu"):
            y = head.linear(table(x.to(dtype), 41, 1), table(w.to(dtype), 12, 1), act=act).float().cpu()
            assert torch.isnan(y[3]).all()
            assert (y[5] == float("inf")).all() if act in ("none", "relu") else not torch.isfinite(y[5]).any() or (y[5] > 1e30).all()
            ok = [i for i in range(40) if i not in (3, 5)]
            assert torch.isfinite(y[ok]).all()


# ------------------------------------------------------------------------------------ log probabilities
def probs_ref(x, t, scale, top):
    z = x.double() * scale
    lse = torch.logsumexp(z, 1)
    lse[(z == float("inf")).any(1)] = float("nan")           # as documented: infinity minus infinity
    none = lse == -float("inf")
    lp = z - lse[:, None]
    p = lp.exp()
    ent = -(torch.where(p > 0, p * lp, torch.where(torch.isnan(p), p, torch.zeros_like(p)))).sum(1)
    lp = torch.where(none[:, None], torch.full_like(lp, -float("inf")), lp)
    ent = torch.where(none, torch.zeros_like(ent), ent)
    mine = torch.zeros(len(x), dtype=torch.float64)
    for r in range(len(x)):
        if t is not None and 0 <= int(t[r]) < x.shape[1]:
            mine[r] = lp[r, int(t[r])]
    ids = np.zeros((len(x), top), np.int64)
    for r in range(len(x)):
        v = x[r].double().numpy()
        key = np.where(np.isnan(v), np.inf, v + 0.0)
        ids[r] = np.lexsort((np.arange(len(v)), -key, ~np.isnan(v)))[:top]
    ids = torch.from_numpy(ids)
    zmax = torch.where(torch.isfinite(z), z.abs(), torch.zeros_like(z)).amax(1)
    # z rounded once; its exponent t log2 e; chains of at most 128 + C / 256 terms
    e = u * (16 + 128 + x.shape[1] / 256) * (1 + math.log(x.shape[1] + 1) + 4 * zmax)
    return mine, ent, lse, ids, torch.gather(lp, 1, ids), e


def check_probs(x, t, scale, top, dtype, ld=None, off=0):
    got = head.log_probs(table(x, ld, off), None if t is None else t.cuda(), top=top, scale=scale)
    mine, ent, lse, ids, top_lp, e = probs_ref(x, t, scale, top)
    assert torch.equal(got["top_ids"].cpu().long(), ids)
    close(got["lse"], lse, e, F32, "lse")
    close(got["logp"], mine, e, F32, "logp")
    close(got["entropy"], ent, e, F32, "entropy")
    close(got["top_logp"], top_lp, e[:, None], F32, "top_logp")


PROBS_SHAPES = [(1, 1), (3, 2), (2, 3), (5, 7), (1, 8), (70, 9), (3, 16), (100, 41), (257, 47), (1, 64), (33, 100), (129, 172), (5, 256), (9, 511),
                (4, 1024), (3, 1025), (3, 2048), (2, 2049), (2, 5003), (1, 20000), (3, 100_003), (1, 300_001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,classes", PROBS_SHAPES)
def test_log_probs(rows, classes, dtype):
    g = gen(rows * 13 + classes)
    x = (3 * torch.randn(rows, classes, generator=g)).to(dtype)
    t = torch.randint(-1, classes, (rows,), generator=g)
    for top, scale, ld, off, targets in ((min(5, classes), 1.0, classes, 0, t), (min(16, classes), 0.7, classes + 3, 1, t.int()), (0, 2.5, classes, 0, None),
                                         (1, 1.0, classes + 8, 0, t), (min(8, classes), 1.0, classes, 0, torch.full_like(t, classes))):
        check_probs(x, targets, scale, top, dtype, ld, off)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [5, 47, 300, 3000, 70_000])
def test_log_probs_ties_masks_and_special_values(classes, dtype):
    """Few distinct values: every alternative is a tie.  Masked classes, rows with none or one left, NaN, infinities, both zeros."""
    g = gen(classes)
    x = torch.randint(-2, 3, (12, classes), generator=g).float()
    x[x == 1] = -0.0
    x[1, torch.rand(classes, generator=g) < 0.6] = -float("inf")
    x[2] = -float("inf")
    x[3] = -float("inf")
    x[3, classes - 1] = 2.0
    x[4, classes // 2] = float("nan")
    x[5, 0] = float("inf")
    x[6] = float("nan")
    x[7] = 3.0
    x[8] = torch.arange(classes) * 0.001                      # best at the end
    x[9] = -torch.arange(classes) * 0.001
    x[10] = -float(torch.finfo(dtype).max)                    # masks by the type's lowest value
    x[10, 2] = 1.0
    x[11] = -float(torch.finfo(dtype).max)
    x = x.to(dtype)
    t = torch.randint(0, classes, (12,), generator=g)
    t[0] = -1
    check_probs(x, t, 1.0, min(16, classes), dtype)
    check_probs(x, t, 1.0, min(3, classes), dtype, classes + 1, 1)


def probs_grad_ref(x, t, lse, ent, g, h, scale):
    z, lse = x.double() * scale, lse.double()
    none = lse == -float("inf")
    lp = torch.where(none[:, None], torch.full_like(z, -float("inf")), z - lse[:, None])
    p = lp.exp()
    has = (t >= 0) & (t < x.shape[1]) & ~none
    g = torch.where(has, g.double(), torch.zeros(len(x), dtype=torch.float64))[:, None]
    h = torch.where(none, torch.zeros_like(lse), h.double())[:, None]
    flat = torch.where(p > 0, p * (torch.where(p > 0, lp, torch.zeros_like(lp)) + ent.double()[:, None]), p * 0)
    one = torch.zeros_like(z)
    for r in range(len(x)):
        if has[r]:
            one[r, int(t[r])] = 1
    size = p * (g.abs() + h.abs() * (lp.clamp(min=-1e3).abs() + ent.double().abs()[:, None]))
    e_lp = u * (4 * torch.nan_to_num(z, 0, 0, 0).abs() + 4 * torch.nan_to_num(lse, 0, 0, 0).abs()[:, None] + 16)
    return scale * (g * (one - p) - h * flat), scale * (size * e_lp + p * h.abs() * e_lp + 4 * u * (g.abs() * one + size))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,classes", PROBS_SHAPES[:-2] + [(2, 70_001)])
def test_log_probs_backward(rows, classes, dtype):
    g = gen(rows * 7 + classes)
    x = (3 * torch.randn(rows, classes, generator=g)).to(dtype)
    if rows > 2:
        x[1] = -float("inf")
        x[2, ::2] = -float("inf")
    t = torch.randint(-1, classes, (rows,), generator=g)
    for scale, ld, off, tt, use in ((1.0, classes, 0, t, "both"), (0.7, classes + 3, 1, t.int(), "logp"), (2.0, classes, 0, t, "entropy")):
        _, ent, lse, *_ = probs_ref(x, t, scale, 0)
        lse, ent = lse.float(), ent.float()
        gl, ge = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
        got = head.log_probs_backward(table(x, ld, off), tt.cuda(), lse.cuda(), ent.cuda(), g_logp=gl.cuda() if use != "entropy" else None,
                                      g_entropy=ge.cuda() if use != "logp" else None, scale=scale)
        want, e = probs_grad_ref(x, t, lse, ent, gl if use != "entropy" else 0 * gl, ge if use != "logp" else 0 * ge, scale)
        assert got.dtype == dtype
        close(got, want, e, dtype, "dlogits " + use)


def test_log_probs_gradient_against_differences():
    g = gen(9)
    x, t = torch.randn(4, 7, generator=g), torch.tensor([0, 6, -1, 3])
    gl, ge = torch.randn(4, generator=g), torch.randn(4, generator=g)
    out = head.log_probs(x.cuda(), t.cuda(), scale=1.3)
    got = head.log_probs_backward(x.cuda(), t.cuda(), out["lse"], out["entropy"], g_logp=gl.cuda(), g_entropy=ge.cuda(), scale=1.3)

    def loss(x_):
        lp = torch.log_softmax(x_ * 1.3, 1)
        mine = torch.stack([lp[r, int(t[r])] if t[r] >= 0 else lp.new_zeros(()) for r in range(4)])
        return float((mine * gl.double()).sum() - ((lp.exp() * lp).sum(1) * ge.double()).sum())
    differences(loss, [x], [got], 2e-5)


# ------------------------------------------------------------------------------------ all of them
def test_no_rows():
    z = lambda *s: torch.empty(*s, device="cuda")                                            # noqa: E731
    y, mean, rstd = head.layer_norm(z(0, 5))
    assert y.shape == (0, 5) and mean.shape == (0,)
    _, dw, db = head.layer_norm_backward(z(0, 5), z(0, 5), z(0), z(0))
    assert torch.equal(dw, torch.zeros_like(dw)) and torch.equal(db, torch.zeros_like(db))
    assert head.linear(z(0, 5), z(5, 3)).shape == (0, 3)
    dx, dw, db = head.linear_backward(z(0, 3), z(0, 5), z(5, 3))
    assert dx.shape == (0, 5) and torch.equal(dw, torch.zeros(5, 3, device="cuda")) and torch.equal(db, torch.zeros(3, device="cuda"))
    out = head.log_probs(z(0, 4), top=2)
    assert out["top_ids"].shape == (0, 2)
    assert head.log_probs_backward(z(0, 4), None, z(0), g_logp=z(0)).shape == (0, 4)


def test_one_row_for_all_and_other_orders():
    """Rows that are views of one row (a gradient that was broadcast), transposed and column-strided tensors."""
    g = gen(11)
    x = torch.randn(50, 24, generator=g).cuda()
    one = torch.randn(1, 24, generator=g).cuda()
    wide = one.expand(50, 24)
    assert torch.equal(head.layer_norm(wide)[0], head.layer_norm(wide.contiguous())[0])
    w = torch.randn(24, 10, generator=g).cuda()
    a, b = head.linear_backward(wide, wide, x[:24].contiguous()), head.linear_backward(wide.contiguous(), wide.contiguous(), x[:24])
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert torch.equal(head.linear(x.t().contiguous().t(), w.t().contiguous().t()), head.linear(x, w))
    assert torch.equal(head.log_probs(x[:, ::2], top=3)["top_ids"], head.log_probs(x[:, ::2].contiguous(), top=3)["top_ids"])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_offsets_beyond_32_bits(dtype):
    """Rows so far apart that their places pass 2^31 elements (and 2^32 bytes)."""
    rows, ld = 20, (1 << 27) + 5
    flat = torch.empty(rows * ld, dtype=dtype, device="cuda")
    far = flat.as_strided((rows, 128), (ld, 1))
    x = torch.randn(rows, 128, generator=gen(2)).to(dtype).cuda()
    far.copy_(x)
    w = torch.randn(128, 47, generator=gen(4)).to(dtype).cuda()
    assert all(torch.equal(a, b) for a, b in zip(head.layer_norm(far), head.layer_norm(x)))
    assert torch.equal(head.linear(far, w), head.linear(x, w))
    dy = torch.randn(rows, 47, generator=gen(6)).to(dtype).cuda()
    assert all(torch.equal(a, b) for a, b in zip(head.linear_backward(dy, far, w), head.linear_backward(dy, x, w)))
    p, q = head.log_probs(far, top=4), head.log_probs(x, top=4)
    assert all(torch.equal(p[k], q[k]) for k in p)
    mean, rstd = head.layer_norm(x)[1:]
    assert all(torch.equal(a, b) for a, b in zip(head.layer_norm_backward(far, far, mean, rstd), head.layer_norm_backward(x, x, mean, rstd)))


def head_step(x, w, t):
    y, mean, rstd = head.layer_norm(x)
    h, z = head.linear(y, w[0], act="gelu", residual=y, keep_pre=True)
    logits = head.linear(h, w[1])
    out = head.log_probs(logits, t, top=3)
    g = torch.full_like(out["logp"], -1.0 / len(x))
    dl = head.log_probs_backward(logits, t, out["lse"], g_logp=g)
    dh, dw1, _ = head.linear_backward(dl, h, w[1])
    dy, dw0, _ = head.linear_backward(dh, y, w[0], pre=z, act="gelu")
    dx, dg, db = head.layer_norm_backward(dy + dh, x, mean, rstd)
    return [out[k] for k in sorted(out)] + [dw1, dw0, dx, dg, db]


def head_data(dtype, rows=700, classes=47):
    g = gen(21)
    x = torch.randn(rows, 64, generator=g).to(dtype).cuda()
    w = [(torch.randn(64, n, generator=g) / 8).to(dtype).cuda() for n in (64, classes)]
    return x, w, torch.randint(-1, classes, (rows,), generator=g).cuda()


@pytest.mark.parametrize("dtype", TYPES)
def test_same_bits_again_and_on_another_stream(dtype):
    x, w, t = head_data(dtype)
    want = head_step(x, w, t)
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(want, head_step(x, w, t)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x2 = x * 1                          # made on the side stream, used there at once
        got = head_step(x2, w, t)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("classes", [47, 5000])
def test_graph_replays(classes):
    x, w, t = head_data(BF16, classes=classes)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        head_step(x, w, t)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = head_step(x, w, t)
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=gen(100 + i)).to(BF16))
        graph.replay()
        torch.cuda.synchronize()
        want = head_step(x, w, t)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), "replay %d" % i


def test_refusals():
    x = torch.zeros(4, 8, device="cuda")
    w = torch.zeros(8, 3, device="cuda")
    v = torch.zeros(8, device="cuda")
    s = torch.zeros(4, device="cuda")
    for call, error in (
            (lambda: head.layer_norm(x.cpu()), ValueError), (lambda: head.layer_norm(x[0]), ValueError), (lambda: head.layer_norm(x.double()), TypeError),
            (lambda: head.layer_norm(x, v[:7]), ValueError), (lambda: head.layer_norm(x, v.half()), TypeError), (lambda: head.layer_norm(x, v, v.cpu()), ValueError),
            (lambda: head.layer_norm(x, eps=0.0), InkError), (lambda: head.layer_norm(x, eps=float("nan")), InkError),
            (lambda: head.layer_norm(torch.zeros(1, 16385, device="cuda")), InkError), (lambda: head.layer_norm(x[:, :0]), InkError),
            (lambda: head.layer_norm_backward(x, x[:3], s, s), ValueError), (lambda: head.layer_norm_backward(x, x, s[:3], s), ValueError),
            (lambda: head.layer_norm_backward(x.half(), x, s, s), TypeError), (lambda: head.layer_norm_backward(x, x, s, s, v, param_dtype=BF16), TypeError),
            (lambda: head.linear(x, w.t()), ValueError), (lambda: head.linear(x, w.half()), TypeError), (lambda: head.linear(x, w, act="tanh"), ValueError),
            (lambda: head.linear(x, w, residual=x), ValueError), (lambda: head.linear(x, w, out_dtype=BF16), TypeError), (lambda: head.linear(x, w, v), ValueError),
            (lambda: head.linear_backward(x[:, :3], x, w, act="gelu"), ValueError), (lambda: head.linear_backward(x[:, :2], x, w), ValueError),
            (lambda: head.linear_backward(x[:, :3], x.half(), w.half()), TypeError), (lambda: head.linear_backward(x[:, :3].half(), x, w), TypeError),
            (lambda: head.log_probs(x, top=9), ValueError), (lambda: head.log_probs(x, top=-1), ValueError), (lambda: head.log_probs(x, s), TypeError),
            (lambda: head.log_probs(x, s[:3].long()), ValueError), (lambda: head.log_probs(x, scale=0.0), InkError), (lambda: head.log_probs(x, scale=-1.0), InkError),
            (lambda: head.log_probs(torch.zeros(2, 20, device="cuda"), top=17), ValueError),
            (lambda: head.log_probs_backward(x, None, s), InkError), (lambda: head.log_probs_backward(x, None, s, g_entropy=s), InkError),
            (lambda: head.log_probs_backward(x, None, s[:3], g_logp=s), ValueError)):
        with pytest.raises(error) as e:
            call()
        assert str(e.value)
    assert torch.equal(head.linear(x, w), torch.zeros(4, 3, device="cuda")), "a refusal leaves nothing behind"
