"""The operators of an answer head's residual blocks (root-mean-square norm, gated pair of projections) against their formulas in
64 bits, on the CPU.

Tolerances follow from the arithmetic: u = 2^-24 for 32-bit operations, U[type] for the final rounding; a sum whose longest chain of
additions is n terms errs by at most n u times the sum of the magnitudes, to first order.
"""
import math

import pytest
import torch

from paper_2309_11071_amd import head
from test_gpu_head import BF16, CHAIN, F16, F32, TYPES, U, close, differences, gen, table, u

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn
E = 2.0 ** -20
ACTS = ["none", "relu", "gelu", "silu"]
# ------------------------------------------------------------------------------------ root-mean-square norm
SHAPES = [(1, 1), (3, 2), (2, 3), (1, 7), (5, 8), (1, 9), (33, 16), (2, 41), (65, 47), (7, 64), (130, 100), (1, 128), (257, 128), (9, 172),
          (64, 256), (31, 257), (3, 512), (17, 602), (5, 1000), (3, 1024), (2, 1100), (2, 2047), (2, 2049), (1, 4100), (3, 4097), (2, 8192), (2, 8200),
          (1, 16384), (3, 16383)]
EPS = 1e-6
"""A lane adds at most 32 elements, a group's sum at most 16 + 10 more, or 4 more of 256 threads: CHAIN covers them."""


def rms_ref(x, res, w, eps, dtype):
    t = x if res is None else (x.float() + res.float()).to(dtype)          # one 32-bit addition, rounded: as it is stored
    v = t.double()
    rstd = (v.square().mean(1) + eps).rsqrt()
    e_rstd = rstd * (CHAIN * u + 6 * u)                                      # half of the sum's error, division, root, reciprocal
    w = torch.ones(x.shape[1], dtype=torch.float64) if w is None else w.double()
    y = v * rstd[:, None] * w
    return y, t, rstd, y.abs() * (e_rstd / rstd)[:, None] + 3 * u * y.abs(), e_rstd


def values(codes, scale):
    return codes.float().double().cpu() * scale.double().cpu()[:, None]


def step_of(a):
    """Distance of the e4m3 numbers around a."""
    return torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=2.0 ** -6)))) / 8


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_rms_norm(rows, cols, dtype):
    g = gen(rows * 31 + cols)
    x, res = ((torch.randn(rows, cols, generator=g) * 2).to(dtype) for _ in range(2))
    w = (1 + 0.3 * torch.randn(cols, generator=g)).to(dtype)
    for ld, off, pw, pr in ((cols, 0, w, res), (cols + 3, 1, w.float(), None), (cols + 16, 0, None, res), (2 * cols + 1, 3, None, None)):
        tx, tr = table(x, ld, off), None if pr is None else table(pr, ld + 1, off)
        want, t, rstd, e, e_rstd = rms_ref(x, pr, pw, EPS, dtype)
        y, total, r = head.rms_norm(tx, None if pw is None else pw.cuda(), residual=tr)
        assert y.dtype == dtype and (total is tx if pr is None else torch.equal(total.cpu(), t))
        close(y, want, e, dtype, "y")
        close(r, rstd, e_rstd, F32, "rstd")
        codes, scale, total, r8 = head.rms_norm(tx, None if pw is None else pw.cuda(), residual=tr, out_dtype=E4M3)
        assert codes.dtype == E4M3 and torch.equal(r8, r) and (total is tx if pr is None else torch.equal(total.cpu(), t))
        top = want.abs().amax(1)
        close(scale, top / 448, (top * (CHAIN + 10) * u) / 448, F32, "scale")
        # half a step of the codes, and what the 32-bit numbers before the rounding and the scale are off
        s = scale.double().cpu()[:, None]
        off_by = (values(codes, scale) - want).abs()
        tol = step_of(want / s) * s * 0.5 * (1 + E) + e + 4 * u * want.abs() + want.abs() * (CHAIN + 10) * u
        assert (off_by <= tol).all(), float((off_by / tol).max())
        assert codes.float().abs().max() <= 448


def rms_grad_ref(dy, t, rstd, w, dt):
    dy, t, r = dy.double(), t.double(), rstd.double()[:, None]
    w = torch.ones(t.shape[1], dtype=torch.float64) if w is None else w.double()
    h = t * r
    g = dy * w
    along = (g * h).mean(1, keepdim=True)
    dx = r * (g - h * along)
    a_gh = (g * h).abs().mean(1, keepdim=True)
    e = r.abs() * (4 * u * g.abs() + (CHAIN + 10) * u * h.abs() * a_gh)
    if dt is not None:
        dx = dx + dt.double()
        e = e + u * dx.abs()
    return dx, (dy * h).sum(0), e, (len(t) + 64) * u * (dy * h).abs().sum(0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES + [(5000, 47), (3001, 256), (2100, 602), (1500, 1100), (700, 2050), (600, 9000)])
def test_rms_norm_backward(rows, cols, dtype):
    g = gen(rows * 17 + cols)
    t, dy, dt = ((torch.randn(rows, cols, generator=g) * 2).to(dtype) for _ in range(3))
    w = (1 + 0.3 * torch.randn(cols, generator=g)).to(dtype)
    rstd = (t.float().square().mean(1) + EPS).rsqrt()
    for ld, off, pw, pt in ((cols, 0, w, dt), (cols + 5, 1, w.float(), None), (cols + 2, 2, None, dt)):
        dx, dw = head.rms_norm_backward(table(dy, ld, off), table(t, ld + 1, off), rstd.cuda(), None if pw is None else pw.cuda(),
                                        d_total=None if pt is None else table(pt, ld + 2, off))
        want = rms_grad_ref(dy, t, rstd, pw, pt)
        p = dtype if pw is None else pw.dtype
        assert dw.dtype == p
        close(dx, want[0], want[2], dtype, "dx")
        close(dw, want[1], want[3], p, "dweight")
    dx2, none = head.rms_norm_backward(dy.cuda(), t.cuda(), rstd.cuda(), need_dweight=False)
    assert none is None and torch.equal(dx2, head.rms_norm_backward(dy.cuda(), t.cuda(), rstd.cuda())[0])
    none, dw = head.rms_norm_backward(dy.cuda(), t.cuda(), rstd.cuda(), need_dx=False, param_dtype=F32)
    want = rms_grad_ref(dy, t, rstd, None, None)
    assert none is None
    close(dw, want[1], want[3], F32, "dweight alone")


def test_rms_norm_gradient_against_differences():
    """Central differences of the formula in 64 bits (step 1e-5: truncation and rounding below 1e-8); a residual's gradient is the same."""
    g = gen(3)
    x, res, dy, dt, w = (torch.randn(3, 11, generator=g) for _ in range(5))
    w = w[0]
    y, total, rstd = head.rms_norm(x.cuda(), w.cuda(), residual=res.cuda())
    dx, dw = head.rms_norm_backward(dy.cuda(), total, rstd, w.cuda(), d_total=dt.cuda())

    def loss(x_, r_, w_):
        t = x_.double() + r_.double()
        y = t * (t.square().mean(1, keepdim=True) + EPS).rsqrt() * w_.double()
        return float((y * dy.double() + t * dt.double()).sum())
    differences(loss, [x, res, w], [dx, dx, dw], 2e-5)


def test_rms_norm_of_no_rows_zeros_and_numbers_that_are_none():
    y, total, rstd = head.rms_norm(torch.empty(0, 5, device="cuda"), residual=torch.empty(0, 5, device="cuda"))
    assert y.shape == total.shape == (0, 5) and rstd.shape == (0,)
    codes, scale, _, _ = head.rms_norm(torch.empty(0, 5, device="cuda"), out_dtype=E4M3)
    assert codes.shape == (0, 5) and scale.shape == (0,)
    dx, dw = head.rms_norm_backward(torch.empty(0, 5, device="cuda"), torch.empty(0, 5, device="cuda"), torch.empty(0, device="cuda"))
    assert dx.shape == (0, 5) and torch.equal(dw.cpu(), torch.zeros(5))
    x = torch.zeros(5, 40)
    x[1, 3], x[2, 7], x[3, 0] = float("nan"), float("inf"), 1e-30
    x[4] = 3
    codes, scale, total, rstd = head.rms_norm(x.cuda(), out_dtype=E4M3)
    assert scale[0] == 0 and not codes[0].float().any(), "a row of zeros"
    for row in (1, 2):
        assert torch.isnan(scale[row]) and torch.isnan(codes[row].float()).all()
    assert torch.equal(codes[4].float().cpu(), torch.full((40,), 448.0))
    y = head.rms_norm(x.cuda())[0].cpu()
    assert torch.isnan(y[1]).all() and torch.isnan(y[2, 7]) and not y[2, :7].any() and not y[0].any()
    w = torch.full((40,), 1e-38)
    codes, scale, _, _ = head.rms_norm(x[4:].cuda(), w.cuda(), out_dtype=E4M3)
    assert scale[0] == 0 and not codes.float().any(), "below the smallest scale"


def test_rms_norm_broadcast_rows():
    """ld 0: one row for all, as an expanded tensor has it."""
    row = torch.randn(1, 70, generator=gen(1)).cuda()
    y, total, rstd = head.rms_norm(row.expand(9, 70), residual=row.expand(9, 70))
    one = head.rms_norm(row, residual=row)
    assert torch.equal(y, one[0].expand(9, 70)) and torch.equal(total, one[1].expand(9, 70)) and torch.equal(rstd, one[2].expand(9))


# ------------------------------------------------------------------------------------ gated pair
def cdf(z, act):
    """F of act(z) = z F(z), and its slope."""
    if act == "none":
        return torch.ones_like(z), torch.zeros_like(z)
    if act == "relu":
        return (z > 0).double(), torch.zeros_like(z)
    if act == "gelu":
        return torch.special.ndtr(z), torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.sigmoid(z), torch.sigmoid(z) * torch.sigmoid(-z)


# how far the 32-bit activations and slopes are from the formulas, relative to 1 + |z| (a polynomial of 1.5e-7 for gelu; exponential,
# reciprocal and some roundings otherwise)
E_ACT = {"none": 0.0, "relu": 0.0, "gelu": 6e-7, "silu": 6e-7}


def lost(x, w):
    """What the 8-bit matrix instructions drop of 64 products each: of every one up to 2^-14 of the largest."""
    e = torch.zeros(x.shape[0], w.shape[1], dtype=torch.float64)
    for k in range(0, x.shape[1], 64):
        for r in range(x.shape[0]):
            e[r] += 64 * 2.0 ** -14 * (x[r, k:k + 64, None] * w[k:k + 64]).abs().amax(0)
    return e


def gated_ref(x, wg, wu, act, terms, more=None):
    """h, its error bound; x and the weights in 64 bits.  terms: the longest chain of a sum."""
    g, u_ = x @ wg, x @ wu
    eg, eu = (terms + 4) * u * (x.abs() @ wg.abs()), (terms + 4) * u * (x.abs() @ wu.abs())
    if more is not None:
        eg, eu = eg + more[0], eu + more[1]
    f, df = cdf(g, act)
    a = g * f
    slope = (f + g * df).abs() + eg                               # curvature at most 1
    if act in ("relu", "none"):
        slope = torch.ones_like(g)                                # either side of the corner
    ea = slope * eg + eg * eg + E_ACT[act] * (1 + g.abs())
    h = a * u_
    return h, ea * u_.abs() + (a.abs() + ea) * eu + u * h.abs()


GATED = [(1, 1, 1), (1, 5, 3), (3, 8, 8), (2, 16, 33), (17, 31, 64), (1, 128, 341), (16, 64, 171), (17, 64, 172), (130, 47, 65), (129, 128, 100), (300, 100, 267),
         (64, 256, 683), (33, 602, 130), (257, 129, 31), (1, 1030, 70), (40, 700, 9), (1000, 65, 344)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,hidden", GATED)
def test_gated(rows, cols, hidden, dtype):
    g = gen(rows * 7 + cols * 3 + hidden)
    x = torch.randn(rows, cols, generator=g).to(dtype)
    wg, wu = ((torch.randn(cols, hidden, generator=g) * cols ** -0.5).to(dtype) for _ in range(2))
    for i, act in enumerate(ACTS):
        ld, off = cols + (0, 3, 16, 1)[i], (0, 1, 0, 3)[i]
        h = head.gated(table(x, ld, off), table(wg, hidden + off, off), table(wu, hidden + 2 * off, off), act=act)
        want, e = gated_ref(x.double(), wg.double(), wu.double(), act, cols)
        close(h, want, e, dtype, act)
    if hidden > 1:                                                # both in one matrix, as a checkpoint may have them
        both = torch.cat([wg, wu], 1).cuda()
        assert torch.equal(head.gated(x.cuda(), both[:, :hidden], both[:, hidden:], act="silu"), head.gated(x.cuda(), wg.cuda(), wu.cuda(), act="silu"))


def to_codes(x, dim):
    scale = x.abs().amax(dim, keepdim=True) / 448
    return (x / scale.clamp(min=1e-30)).to(E4M3), scale.squeeze(dim)


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("rows,cols,hidden", GATED)
def test_gated_of_8_bits(rows, cols, hidden, out):
    g = gen(rows * 5 + cols * 3 + hidden)
    x, xs = to_codes(torch.randn(rows, cols, generator=g), 1)
    wg, sg = to_codes(torch.randn(hidden, cols, generator=g) * cols ** -0.5, 1)
    wu, su = to_codes(torch.randn(hidden, cols, generator=g) * cols ** -0.5, 1)
    dx, dg, du = x.double() * xs.double()[:, None], (wg.double() * sg.double()[:, None]).t(), (wu.double() * su.double()[:, None]).t()
    flat = torch.zeros(3 + rows * (cols + 5), dtype=torch.uint8, device="cuda").view(E4M3)
    apart = flat[3:].as_strided((rows, cols), (cols + 5, 1))
    apart.copy_(x.cuda())
    scales = dict(x_scale=xs.cuda(), gate_scale=sg.cuda(), up_scale=su.cuda())
    for i, act in enumerate(ACTS):
        h = head.gated(apart if i % 2 else x.cuda(), wg.cuda().t(), wu.cuda().t(), act=act, out_dtype=out, **scales)
        want, e = gated_ref(dx, dg, du, act, cols, None if out is F32 else (lost(dx, dg), lost(dx, du)))
        close(h, want, e, out, act)
    assert torch.equal(h, head.gated(x.cuda(), wg.cuda().t().contiguous(), wu.cuda().t().contiguous(), act=act, out_dtype=out, **scales)), "rows of weights are turned"
    assert head.gated(x.cuda(), wg.cuda().t(), wu.cuda().t(), **scales).dtype == BF16


def gated_grad_ref(dh, x, wg, wu, act, dtype):
    """Gradients and their bounds: dg and du err by the projections' error, and with 16 bits by their rounding."""
    rows, cols = x.shape
    dh, x, wg, wu = dh.double(), x.double(), wg.double(), wu.double()
    g, u_ = x @ wg, x @ wu
    eg, eu = (cols + 4) * u * (x.abs() @ wg.abs()), (cols + 4) * u * (x.abs() @ wu.abs())
    f, df = cdf(g, act)
    a, s = g * f, f + g * df
    dg, du = dh * u_ * s, dh * a
    jump = eg * 1.0
    if act == "relu":
        jump = (g.abs() <= eg).double()                           # at the corner either slope
    elif act == "none":
        jump = torch.zeros_like(g)
    e_slope = jump + E_ACT[act] * (1 + g.abs())
    e_dg = dh.abs() * (eu * s.abs() + u_.abs() * e_slope) + 4 * u * dg.abs()
    slope = s.abs() + eg if act in ("gelu", "silu") else torch.ones_like(g)
    e_du = dh.abs() * (slope * eg + E_ACT[act] * (1 + g.abs())) + 4 * u * du.abs()
    if dtype is not F32 and not (rows * wg.shape[1] <= 65536 if rows <= 32 else rows <= 64 and rows * wg.shape[1] <= 4096):   # (few: kept in 32 bits)
        tiny = 2.0 ** -25 if dtype is F16 else 0.0
        e_dg, e_du = e_dg + U[dtype] * (dg.abs() + e_dg) + tiny, e_du + U[dtype] * (du.abs() + e_du) + tiny
    n, m = 2 * wg.shape[1] + 16, rows + 64
    dx, e_dx = dg @ wg.t() + du @ wu.t(), e_dg @ wg.abs().t() + e_du @ wu.abs().t() + n * u * (dg.abs() @ wg.abs().t() + du.abs() @ wu.abs().t())
    return ((dx, e_dx), (x.t() @ dg, x.abs().t() @ e_dg + m * u * (x.abs().t() @ dg.abs())),
            (x.t() @ du, x.abs().t() @ e_du + m * u * (x.abs().t() @ du.abs())))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,hidden", GATED)
def test_gated_backward(rows, cols, hidden, dtype):
    g = gen(rows * 11 + cols * 3 + hidden)
    x, dh = torch.randn(rows, cols, generator=g).to(dtype), torch.randn(rows, hidden, generator=g).to(dtype)
    wg, wu = ((torch.randn(cols, hidden, generator=g) * cols ** -0.5).to(dtype) for _ in range(2))
    for i, act in enumerate(ACTS):
        off = (0, 1, 0, 3)[i]
        args = (table(dh, hidden + off, off), table(x, cols + off, off), table(wg, hidden + 2 * off, off), table(wu, hidden + off, off))
        got = head.gated_backward(*args, act=act)
        for a, (want, e), name in zip(got, gated_grad_ref(dh, x, wg, wu, act, dtype), ("dx", "dw_gate", "dw_up")):
            assert a.dtype == dtype
            close(a, want, e, dtype, "%s %s" % (act, name))
    dx, none, none2 = head.gated_backward(*args, act=act, need_dweights=False)
    assert none is none2 is None and torch.equal(dx, got[0])
    none, dg, du = head.gated_backward(*args, act=act, need_dx=False)
    assert none is None and torch.equal(dg, got[1]) and torch.equal(du, got[2])
    assert head.gated_backward(*args, act=act, need_dx=False, need_dweights=False) == (None, None, None)


# enough rows for the kernels that keep the weights in registers, or for their fallback (deep sums, few columns): every class of depth and
# width, sizes beside the tiles', last tiles of one row, rows that no workgroup shares with another
MANY = [(32768, 64, 32, 0), (32769, 128, 344, 3), (33000, 47, 31, 1), (32800, 100, 64, 2), (32769, 65, 172, 3), (32801, 8, 341, 0), (32790, 120, 130, 1),
        (32777, 256, 100, 3), (33333, 250, 41, 2), (32769, 200, 300, 3), (32801, 7, 40, 1), (32769, 270, 50, 3), (32770, 33, 7, 2), (36000, 129, 8, 3), (16385, 200, 70, 2)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,hidden,act", MANY)
def test_gated_of_many_rows(rows, cols, hidden, act, dtype):
    g = gen(rows + cols * 3 + hidden)
    x, dh = torch.randn(rows, cols, generator=g).to(dtype), torch.randn(rows, hidden, generator=g).to(dtype)
    wg, wu = ((torch.randn(cols, hidden, generator=g) * cols ** -0.5).to(dtype) for _ in range(2))
    off = hidden % 4
    args = (table(x, cols + off, off), table(wg, hidden + 2 * off, off), table(wu, hidden + off, off))
    h = head.gated(*args, act=ACTS[act])
    want, e = gated_ref(x.double(), wg.double(), wu.double(), ACTS[act], cols)
    close(h, want, e, dtype, "h")
    got = head.gated_backward(table(dh, hidden + off, off), *args, act=ACTS[act])
    for a, (want, e), name in zip(got, gated_grad_ref(dh, x, wg, wu, ACTS[act], dtype), ("dx", "dw_gate", "dw_up")):
        close(a, want, e, dtype, name)
    view = torch.full((rows, hidden + 9), 7.0, dtype=dtype, device="cuda")   # results as columns of a wider table: nothing beside them is written
    lib, stream, t = head._functions(), torch.cuda.current_stream().cuda_stream, head.TYPES[dtype]
    xd, gd, ud = x.cuda(), wg.cuda(), wu.cuda()
    assert lib.ink_gated(xd.data_ptr(), cols, None, gd.data_ptr(), hidden, ud.data_ptr(), hidden, None, None, rows, cols, hidden, t, t, act,
                         view[:, 4:].data_ptr(), hidden + 9, stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(view[:, 4:4 + hidden], h), "the layout of the tensors changed the result"
    assert (view[:, :4] == 7).all() and (view[:, 4 + hidden:] == 7).all()


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("rows,cols,hidden,act", [(32769, 256, 130, 2), (33000, 128, 344, 3), (32801, 100, 31, 1), (32770, 16, 64, 0), (32769, 500, 70, 3), (32800, 520, 33, 1),
                                                  (32768, 15, 40, 3), (32769, 193, 5, 2)])
def test_gated_of_many_8_bit_rows(rows, cols, hidden, act, out):
    g = gen(rows + cols * 3 + hidden)
    x, xs = to_codes(torch.randn(rows, cols, generator=g), 1)
    wg, sg = to_codes(torch.randn(hidden, cols, generator=g) * cols ** -0.5, 1)
    wu, su = to_codes(torch.randn(hidden, cols, generator=g) * cols ** -0.5, 1)
    dx, dg, du = x.double() * xs.double()[:, None], (wg.double() * sg.double()[:, None]).t(), (wu.double() * su.double()[:, None]).t()
    h = head.gated(x.cuda(), wg.cuda().t(), wu.cuda().t(), act=ACTS[act], out_dtype=out, x_scale=xs.cuda(), gate_scale=sg.cuda(), up_scale=su.cuda())
    # of every product of a row and a column at most its largest factors'
    more = None if out is F32 else tuple(cols * 2.0 ** -14 * dx.abs().amax(1)[:, None] * w.abs().amax(0) for w in (dg, du))
    want, e = gated_ref(dx, dg, du, ACTS[act], cols, more)
    close(h, want, e, out, "h")


def test_gated_gradient_against_differences():
    g = gen(4)
    x, dh = torch.randn(5, 7, generator=g), torch.randn(5, 6, generator=g)
    wg, wu = torch.randn(7, 6, generator=g), torch.randn(7, 6, generator=g)
    for act in ("none", "gelu", "silu"):
        got = head.gated_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), act=act)

        def loss(x_, wg_, wu_):
            z = x_.double() @ wg_.double()
            return float((z * cdf(z, act)[0] * (x_.double() @ wu_.double()) * dh.double()).sum())
        differences(loss, [x, wg, wu], got, 5e-5)


def test_gated_of_no_rows_and_numbers_that_are_none():
    e = torch.empty(0, 6, device="cuda")
    w = torch.randn(6, 5, generator=gen(1)).cuda()
    assert head.gated(e, w, w).shape == (0, 5)
    dx, dg, du = head.gated_backward(torch.empty(0, 5, device="cuda"), e, w, w)
    assert dx.shape == (0, 6) and not dg.any() and not du.any()
    x = torch.randn(200, 6, generator=gen(2)).to(BF16)
    x[150, 2], x[151, 3] = float("nan"), float("inf")
    for rows in (slice(0, 200), slice(150, 152)):
        h = head.gated(x[rows].cuda(), w.to(BF16), w.to(BF16), act="silu").float().cpu()
        bad = ~torch.isfinite(h).all(1)
        assert torch.equal(bad, ~torch.isfinite(x[rows].float()).all(1)), "other rows are untouched"
        dx = head.gated_backward(torch.ones(len(h), 5, device="cuda", dtype=BF16), x[rows].cuda(), w.to(BF16), w.to(BF16))[0]
        assert torch.equal(~torch.isfinite(dx.float().cpu()).all(1), bad)


def test_more_rows_than_one_launch_takes():
    """2^21 rows a launch in tiles (a depth that the registers do not hold), with scales of 8-bit rows beside them."""
    rows, cols, hidden = 2 ** 21 + 100, 264, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, cols, device="cuda", generator=g).to(BF16)
    wg, wu = ((torch.randn(cols, hidden, device="cuda", generator=g) * cols ** -0.5).to(BF16) for _ in range(2))
    h = head.gated(x, wg, wu)
    some = torch.cat([torch.arange(0, 50), torch.arange(2 ** 21 - 50, rows)])
    want, e = gated_ref(x[some.cuda()].double().cpu(), wg.double().cpu(), wu.double().cpu(), "silu", cols)
    close(h[some.cuda()], want, e, BF16, "bf16")
    x8, s8 = to_codes(x.float(), 1)
    w8, sw = to_codes(wg.float().t(), 1)
    h = head.gated(x8, w8.t(), w8.t(), x_scale=s8, gate_scale=sw, up_scale=sw, out_dtype=F32)
    dx, dw = x8[some.cuda()].double().cpu() * s8[some.cuda()].double().cpu()[:, None], (w8.double() * sw.double()[:, None]).t().cpu()
    want, e = gated_ref(dx, dw, dw, "silu", cols)
    close(h[some.cuda()], want, e, F32, "e4m3")


def test_gradient_of_several_parts():
    """dg and du of 2 x 1024 columns: 262144 rows a part, three parts."""
    rows, cols, hidden = 2 * 262144 + 77, 16, 1024
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dh = torch.randn(rows, cols, device="cuda", generator=g).to(BF16), torch.randn(rows, hidden, device="cuda", generator=g).to(BF16)
    wg, wu = ((torch.randn(cols, hidden, device="cuda", generator=g) * cols ** -0.5).to(BF16) for _ in range(2))
    got = head.gated_backward(dh, x, wg, wu)
    for a, (want, e), name in zip(got, gated_grad_ref(dh, x, wg, wu, "silu", BF16), ("dx", "dw_gate", "dw_up")):
        close(a, want.cpu(), e.cpu(), BF16, name)
    again = head.gated_backward(dh, x, wg, wu)
    assert all(torch.equal(a, b) for a, b in zip(got, again)), "the same call gives the same bits"


def test_another_stream_and_a_captured_call():
    """The calls run on the current stream and can be captured; every replay gives what an eager call gives."""
    g = gen(6)
    x, res, dh = (torch.randn(n, 48, generator=g).to(BF16).cuda() for n in (700, 700, 700))
    wg, wu = ((torch.randn(48, 48, generator=g) / 7).to(BF16).cuda() for _ in range(2))

    def call():
        y, total, rstd = head.rms_norm(x, wg[0], residual=res)
        codes, scale, _, _ = head.rms_norm(x, wg[0], residual=res, out_dtype=E4M3)
        h = head.gated(y, wg, wu)
        dy, dg, du = head.gated_backward(dh, y, wg, wu)
        return (h, dg, du, scale, codes.view(torch.uint8), *head.rms_norm_backward(dy, total, rstd, wg[0], d_total=dh))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for i in range(3):
        x.copy_(torch.randn(700, 48, generator=g).to(BF16).cuda())
        graph.replay()
        torch.cuda.synchronize()
        want = call()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i
    assert not torch.equal(first[0], out[0])


def test_refusals_of_the_binding():
    x, w = torch.randn(4, 6, device="cuda"), torch.randn(6, 5, device="cuda")
    e = x.to(E4M3)
    w8 = w.to(E4M3)
    one4, one5 = torch.ones(4, device="cuda"), torch.ones(5, device="cuda")
    bad = [
        (TypeError, lambda: head.rms_norm(x, out_dtype=BF16)), (TypeError, lambda: head.rms_norm(x.double())), (ValueError, lambda: head.rms_norm(x, residual=x[:3])),
        (TypeError, lambda: head.rms_norm(x, residual=x.half())), (ValueError, lambda: head.rms_norm(x, one4)), (ValueError, lambda: head.rms_norm(x.clone().requires_grad_())),
        (head.InkError, lambda: head.rms_norm(x, eps=0.0)), (ValueError, lambda: head.rms_norm_backward(x, x, None)), (ValueError, lambda: head.rms_norm_backward(x, x, one5)),
        (ValueError, lambda: head.rms_norm_backward(x, x, one4, d_total=x[:, :5])), (TypeError, lambda: head.rms_norm_backward(x, x, one4, param_dtype=BF16)),
        (ValueError, lambda: head.gated(x, w, w[:, :4])), (TypeError, lambda: head.gated(x, w.half(), w)), (ValueError, lambda: head.gated(x, w, w, act="tanh")),
        (ValueError, lambda: head.gated(x, w, w, x_scale=one4)), (TypeError, lambda: head.gated(x, w, w, out_dtype=BF16)), (ValueError, lambda: head.gated(e, w8, w8)),
        (TypeError, lambda: head.gated(e, w, w, x_scale=one4, gate_scale=one5, up_scale=one5)), (ValueError, lambda: head.gated(e, w8, w8, x_scale=one4, gate_scale=one4, up_scale=one5)),
        (TypeError, lambda: head.gated(e, w8, w8, x_scale=one4, gate_scale=one5, up_scale=one5, out_dtype=E4M3)), (TypeError, lambda: head.gated_backward(e, e, w8, w8)),
        (ValueError, lambda: head.gated_backward(x, x, w, w)), (TypeError, lambda: head.gated_backward(x[:, :5].half(), x, w, w)),
    ]
    for i, (kind, call) in enumerate(bad):
        with pytest.raises(kind):
            call()
            print(i)
    with torch.no_grad():
        head.rms_norm(x.clone().requires_grad_())


def test_8_bit_weights_that_require_a_gradient_raise():
    """As every tensor of these calls: nothing records the call for autograd."""
    x, w, s = torch.zeros(2, 16, device="cuda").to(E4M3), torch.zeros(8, 16, device="cuda").to(E4M3).t(), torch.ones(8, device="cuda")
    wanted = w.detach().requires_grad_()
    for gate, up in ((wanted, w), (w, wanted)):
        with pytest.raises(ValueError):
            head.gated(x, gate, up, x_scale=s[:2], gate_scale=s, up_scale=s)
        with torch.no_grad():
            assert not head.gated(x, gate, up, x_scale=s[:2], gate_scale=s, up_scale=s).any()
