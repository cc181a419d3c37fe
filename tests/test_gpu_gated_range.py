"""The gated pair's gradient of float16 rows where dg and du, which lie between its products, pass float16's range and the results do not,
against the formulas in 64 bits.

Tolerances: as for ordinary numbers (test_gpu_blocks.py), U = 2^-12 of a number for its rounding to float16, and a part of the largest number of
its surroundings for the numbers that come out subnormal: the numbers of a row in 32 columns (a block's row) are held so that the largest of them
is at least 2^-12, of which half a subnormal step, 2^-25, is 2^-13; for the sums over rows a block of 32 rows is brought to units in which its largest number
is at least 2^-4, which costs half a step a second time: 2 * 2^-25 / 2^-4 = 2^-20 of it.
"""
import pytest
import torch

from paper_2309_11071_amd import head
from test_gpu_blocks import E_ACT, cdf
from test_gpu_head import F16, U, close, gen, table, u

pytestmark = pytest.mark.gpu
NAMES = ("dx", "dw_gate", "dw_up")


def tops(d, rows):
    """Largest magnitude of each 32 columns, of a row or of 32 rows, at every element."""
    r, h = d.shape
    full = torch.zeros(-(-r // 32) * 32, -(-h // 32) * 32, dtype=d.dtype, device=d.device)
    full[:r, :h] = torch.where(torch.isfinite(d), d.abs(), 0.0)
    b = full.view(full.shape[0] // 32, 32, -1, 32)
    t = b.amax((1, 3), keepdim=True) if rows else b.amax(3, keepdim=True)
    return t.expand_as(b).reshape(full.shape)[:r, :h]


def reference(dh, x, wg, wu, act):
    """(dx, dw_gate, dw_up) with their bounds, and the largest of dg and du."""
    rows, cols = x.shape
    dh, x, wg, wu = dh.double(), x.double(), wg.double(), wu.double()
    g, up = x @ wg, x @ wu
    eg, eu = (cols + 4) * u * (x.abs() @ wg.abs()), (cols + 4) * u * (x.abs() @ wu.abs())
    f, df = cdf(g, act)
    a, s = g * f, f + g * df
    dg, du = dh * up * s, dh * a
    jump = {"relu": (g.abs() <= eg).double(), "none": torch.zeros_like(g)}.get(act, eg)
    slope = torch.ones_like(g) if act in ("relu", "none") else s.abs() + eg
    e_dg = dh.abs() * (eu * s.abs() + up.abs() * (jump + E_ACT[act] * (1 + g.abs()))) + 4 * u * dg.abs()
    e_du = dh.abs() * (slope * eg + E_ACT[act] * (1 + g.abs())) + 4 * u * du.abs()
    e_dg, e_du = e_dg + U[F16] * (dg.abs() + e_dg), e_du + U[F16] * (du.abs() + e_du)
    row_g, row_u = (e + 2.0 ** -13 * 1.001 * tops(d, False) for e, d in ((e_dg, dg), (e_du, du)))
    all_g, all_u = (e + 2.0 ** -20 * 1.001 * tops(d, True) for e, d in ((e_dg, dg), (e_du, du)))
    n, m = 2 * wg.shape[1] + 16, rows + 64
    dx = dg @ wg.t() + du @ wu.t(), row_g @ wg.abs().t() + row_u @ wu.abs().t() + n * u * (dg.abs() @ wg.abs().t() + du.abs() @ wu.abs().t())
    return (dx, (x.t() @ dg, x.abs().t() @ all_g + m * u * (x.abs().t() @ dg.abs())),
            (x.t() @ du, x.abs().t() @ all_u + m * u * (x.abs().t() @ du.abs()))), float(torch.maximum(dg.abs(), du.abs()).max())


# tiles and few columns, tiles of dx by 128, sums by 256, both depths of the stream, rows short of a piece, ends of blocks of every kind
SHAPES = [(100, 600, 40), (65, 300, 31), (129, 60, 97), (2000, 520, 70), (9000, 100, 65), (300, 5, 33), (200, 50, 7), (32801, 120, 70), (33000, 60, 31), (16500, 250, 33), (9001, 300, 130)]


@pytest.mark.parametrize("act", ["silu", "gelu", "relu", "none"])
@pytest.mark.parametrize("rows,cols,hidden", [s for s in SHAPES if s[1] >= 40])
def test_beyond_the_largest_number(rows, cols, hidden, act):
    """x and the weights so small that g and u are some 2.4: with gradients of up to 35000, one in a row and a column, dg passes 65504, its products with x and
    the weights do not."""
    g = gen(rows + cols + hidden)
    size = (2.4 / cols) ** 0.5
    x, wg, wu = ((size * (1 + 0.2 * torch.randn(*s, generator=g))).to(F16) for s in ((rows, cols), (cols, hidden), (cols, hidden)))
    n = min(rows, hidden) // 2
    at, column = torch.randperm(rows, generator=g)[:2 * n], torch.randperm(hidden, generator=g)[:n]
    dh = torch.zeros(rows, hidden)
    dh[at[:n], column] = (torch.rand(n, generator=g) * 25000 + 10000) * (torch.randint(0, 2, (n,), generator=g) * 2 - 1)
    dh[at[0], column[0]] = 35000
    dh[at[n:]] = torch.randn(n, hidden, generator=g) * torch.exp2(torch.randint(-16, 1, (n, 1), generator=g).float())       # beside rows of ordinary and of small numbers
    dh = dh.to(F16)
    want, top = reference(dh, x, wg, wu, act)
    assert top > 65504 * 1.1 and all(float(w.abs().max()) < 65000 for w, _ in want), "the case is meant to have results in range"
    off = hidden % 3
    got = head.gated_backward(table(dh, hidden + off, off), table(x, cols + 1, 1), table(wg, hidden, 0), table(wu, hidden + 2, off), act=act)
    for a, (w, e), name in zip(got, want, NAMES):
        close(a, w, e, F16, name)


@pytest.mark.parametrize("scale", [2.0 ** -24, 2.0 ** -20, 2.0 ** -13])
@pytest.mark.parametrize("rows,cols,hidden", SHAPES)
def test_below_the_smallest_number(rows, cols, hidden, scale):
    """Gradients of the size of float16's smallest numbers, as the mean over many rows leaves them: 2^-24 times a number below 1 is 0 in float16, a sum of many
    is not, nor is its product with a large weight."""
    g = gen(rows * 3 + cols + hidden)
    x = (0.01 + 0.01 * torch.rand(rows, cols, generator=g)).to(F16)
    wg, wu = ((30 * torch.randn(cols, hidden, generator=g) * cols ** -0.5).to(F16) for _ in range(2))
    dh = (scale * torch.randint(-3, 4, (rows, hidden), generator=g)).to(F16)
    want, top = reference(dh, x, wg, wu, "silu")
    got = head.gated_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), act="silu")
    for a, (w, e), name in zip(got, want, NAMES):
        close(a, w, e, F16, name)


@pytest.mark.parametrize("rows,cols,hidden", SHAPES)
def test_sizes_that_differ_from_row_to_row_and_column_to_column(rows, cols, hidden):
    """Rows of the gradient and columns of the weights by powers of two apart: a row's dx has the precision of its own numbers, whatever its neighbours hold."""
    g = gen(rows * 5 + cols + hidden)
    x = (torch.randn(rows, cols, generator=g) * cols ** -0.5).to(F16)
    wide = torch.exp2(torch.randint(-10, 5, (hidden,), generator=g).float())
    wg, wu = (torch.randn(cols, hidden, generator=g).to(F16), (torch.randn(cols, hidden, generator=g) * wide).to(F16))
    dh = (torch.randn(rows, hidden, generator=g) * torch.exp2(torch.randint(-24, 8, (rows, 1), generator=g).float())).to(F16)
    want, _ = reference(dh, x, wg, wu, "gelu")
    got = head.gated_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), act="gelu")
    inside = [w.abs() + e < 65504 for w, e in want]
    for a, (w, e), ok, name in zip(got, want, inside, NAMES):
        assert ok.float().mean() > 0.9, name
        close(torch.where(ok.cuda(), a, 0), torch.where(ok, w, 0), e, F16, name)


@pytest.mark.parametrize("rows,cols,hidden", [(200, 64, 100), (9000, 100, 65), (32801, 120, 70)])
def test_a_row_that_passes_all_bounds_leaves_the_others_alone(rows, cols, hidden):
    """Rows with an infinity, a NaN or numbers whose dx is beyond float16: dx of every other row has the bits that it has without them."""
    g = gen(rows)
    x, dh = torch.randn(rows, cols, generator=g).to(F16), torch.randn(rows, hidden, generator=g).to(F16)
    wg, wu = ((torch.randn(cols, hidden, generator=g) * cols ** -0.5).to(F16) for _ in range(2))
    calm = head.gated_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda())[0].cpu()
    bad = [5, 38, 70, rows - 1]
    dh[5, 3], dh[38, 2], x[rows - 1, 1] = float("inf"), float("nan"), float("nan")
    x[70], dh[70] = 60000, 60000
    dx = head.gated_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda())[0].cpu()
    good = torch.ones(rows, dtype=torch.bool)
    good[bad] = False
    assert torch.equal(dx[good], calm[good])
    assert not torch.isfinite(dx[bad]).all(1).any()


def test_parts_of_different_sizes():
    """Three parts of the rows whose gradients lie 2^20 apart: the sums go on from part to part."""
    rows, cols, hidden = 2 * 262144 + 77, 16, 1024
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(rows, cols, device="cuda", generator=g).to(F16)
    wg, wu = ((torch.randn(cols, hidden, device="cuda", generator=g) * cols ** -0.5).to(F16) for _ in range(2))
    for sizes in ((2.0 ** -20, 1.0, 2.0 ** -22), (1.0, 2.0 ** -21, 2.0 ** 5)):
        dh = torch.randn(rows, hidden, device="cuda", generator=g)
        for i, s in enumerate(sizes):
            dh[262144 * i:262144 * (i + 1)] *= s
        dh = dh.to(F16)
        got = head.gated_backward(dh, x, wg, wu)
        want, _ = reference(dh, x, wg, wu, "silu")
        for a, (w, e), name in zip(got, want, NAMES):
            close(a, w.cpu(), e.cpu(), F16, name)
        again = head.gated_backward(dh, x, wg, wu)
        assert all(torch.equal(a, b) for a, b in zip(got, again)), "the same call gives the same bits"
        del want


def test_captured():
    """Replays with gradients of other sizes than the captured call's."""
    g = gen(6)
    x, wg, wu = torch.randn(700, 48, generator=g).to(F16).cuda(), (torch.randn(48, 100, generator=g) / 7).to(F16).cuda(), (torch.randn(48, 100, generator=g) / 7).to(F16).cuda()
    dh = torch.randn(700, 100, generator=g).to(F16).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        head.gated_backward(dh, x, wg, wu)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = head.gated_backward(dh, x, wg, wu)
    for scale in (1.0, 2.0 ** -18, 2.0 ** 4, 2.0 ** -10):
        dh.copy_((torch.randn(700, 100, generator=g) * scale).to(F16))
        graph.replay()
        torch.cuda.synchronize()
        want = head.gated_backward(dh, x, wg, wu)
        assert all(torch.equal(a, b) for a, b in zip(out, want)), scale
