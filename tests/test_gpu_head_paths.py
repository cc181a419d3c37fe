"""Sizes that take the forms of an answer head's operators which small tests do not reach: a wave a row of long rows of logits, tiles below
the row count of the stream, and row loops that take a second turn."""
import math

import pytest
import torch

from paper_2309_11071_amd import head
from test_gpu_head import BF16, F16, F32, TYPES, close, gen, linear_case, linear_grad_ref, linear_ref, norm_grad_ref, norm_ref, table, u

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------ layer norm
def in_range(want, dtype):
    """want with infinity in place of what rounds to it in dtype (sums over all rows pass float16's range)."""
    return torch.where(want.to(dtype).double().abs() == math.inf, want.to(dtype).double(), want)


# rows beyond what one turn of the largest launch takes, for groups of 4, 8, 16, 32 and 64 lanes
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(140_001, 47), (70_001, 128), (33_001, 300), (17_001, 602), (9_001, 1024)])
def test_layer_norm_takes_rows_in_several_turns(rows, cols, dtype):
    g = gen(rows)
    x, dy = ((torch.randn(rows, cols, generator=g) * 2 + 1).to(dtype) for _ in range(2))
    w, b = (1 + 0.3 * torch.randn(cols, generator=g)).to(dtype), torch.randn(cols, generator=g).to(dtype)
    y, mean, rstd = head.layer_norm(x.cuda(), w.cuda(), b.cuda())
    want = norm_ref(x, w, b, 1e-5)
    close(y, want[0], want[3], dtype, "y")
    close(mean, want[1], want[4], F32, "mean")
    close(rstd, want[2], want[5], F32, "rstd")
    mean, rstd = want[1].float(), want[2].float()
    dx, dw, db = head.layer_norm_backward(dy.cuda(), x.cuda(), mean.cuda(), rstd.cuda(), w.cuda())
    want = norm_grad_ref(dy, x, mean, rstd, w)
    close(dx, want[0], want[3], dtype, "dx")
    close(dw, in_range(want[1], dtype), want[4], dtype, "dweight")
    close(db, in_range(want[2], dtype), want[5], dtype, "dbias")


# ------------------------------------------------------------------------------------ linear
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,out", [(20_000, 256, 256), (32_767, 64, 700), (32_700, 128, 48), (32_700, 700, 48), (8_200, 513, 511)])
def test_linear_in_tiles(rows, cols, out, dtype):
    """Fewer rows than the stream takes, 256 tiles and more."""
    g, x, w, b = linear_case(rows, cols, out, dtype, rows + cols + out)
    for act, f32, pad in (("gelu", False, 0), ("none", True, 3)):
        to = F32 if f32 else dtype
        r = torch.randn(rows, out, generator=g).to(to)
        y, z = head.linear(table(x, cols + pad, pad), table(w, out + pad, pad), b.cuda(), act=act, residual=table(r, out + pad, pad), keep_pre=True, out_dtype=to)
        want = linear_ref(x, w, b, act, r)
        close(z, want[1], want[3], to, "z " + act)
        close(y, want[0], want[2], to, "y " + act)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,out", [(64, 300, 1024), (64, 300, 1025), (4, 200, 16384), (5, 200, 16384), (2, 4100, 4100), (61, 1030, 5000)])
def test_linear_of_few_rows_and_wide_results(rows, cols, out, dtype):
    """Beside the number of results up to which rows are taken one by one, and far beyond it."""
    g, x, w, b = linear_case(rows, cols, out, dtype, rows + cols + out)
    r = torch.randn(rows, out, generator=g).to(dtype)
    y, z = head.linear(table(x, cols + 1, 1), table(w, out + 3, 1), b.cuda(), act="silu", residual=table(r, out + 1, 1), keep_pre=True)
    want = linear_ref(x, w, b, "silu", r)
    close(z, want[1], want[3], dtype, "z")
    close(y, want[0], want[2], dtype, "y")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,out", [(20_000, 256, 256), (32_700, 48, 700), (8_200, 513, 511)])
def test_linear_backward_in_tiles(rows, cols, out, dtype):
    g, x, w, _ = linear_case(rows, cols, out, dtype, rows * 3 + cols + out)
    dy, pre = torch.randn(rows, out, generator=g), 2 * torch.randn(rows, out, generator=g)
    for act, to, pad in (("none", dtype, 1), ("gelu", dtype, 0)) + ((("silu", F32, 2), ("none", F32, 0)) if dtype == BF16 else ()):
        d, p = dy.to(to), pre.to(to)
        got = head.linear_backward(table(d, out + pad, pad), table(x, cols + pad, pad), table(w, out + pad, pad),
                                   pre=None if act == "none" else table(p, out + pad, pad), act=act)
        want = linear_grad_ref(d, x, w, p, act, dtype)
        for i, name in enumerate(("dx", "dweight", "dbias")):
            close(got[i], want[i], want[3 + i], dtype, "%s %s %s" % (name, act, to))


# ------------------------------------------------------------------------------------ log probabilities
def check(x, t, top, dtype, ld=None, off=0):
    """head.log_probs of x (on the GPU) against its definition in 64 bits, every row."""
    rows, classes = x.shape
    got = head.log_probs(x if ld is None else table(x, ld, off), t, top=top)
    ids = torch.sort(torch.where(x == 0, torch.zeros_like(x), x), dim=1, descending=True, stable=True).indices[:, :top]      # NaN first
    assert torch.equal(got["top_ids"].long(), ids)
    z = x.double()
    lse = torch.logsumexp(z, 1)
    lse[(z == float("inf")).any(1)] = float("nan")
    none = lse == -float("inf")
    lp = torch.where(none[:, None], z.new_tensor(-float("inf")), z - lse[:, None])
    p = lp.exp()
    ent = torch.where(none, 0.0, -torch.where(p == 0, 0.0, p * lp).sum(1))
    has = (t >= 0) & (t < classes)
    mine = torch.where(has, lp.gather(1, t.clamp(0, classes - 1)[:, None])[:, 0], 0.0)
    zmax = torch.where(torch.isfinite(z), z.abs(), 0.0).amax(1)
    e = (u * (16 + 128 + classes / 64) * (1 + math.log(classes + 1) + 4 * zmax)).cpu()
    for k, want in (("lse", lse), ("logp", mine), ("entropy", ent), ("top_logp", lp.gather(1, ids))):
        close(got[k], want.cpu(), e[:, None] if k == "top_logp" else e, F32, "%s top %d" % (k, top))


def special(x, g):
    """Ties, masks, rows without a class, NaN and infinities among random rows."""
    n, classes = x.shape
    x[1::7] = torch.randint(-2, 3, x[1::7].shape, generator=g, device="cuda").float()
    x[2::11][torch.rand(x[2::11].shape, generator=g, device="cuda") < 0.6] = -float("inf")
    x[5] = x[n - 1] = -float("inf")
    x[6] = -float("inf")
    x[6, classes - 1] = 2.0
    x[7, classes // 2] = float("nan")
    x[8, 0] = float("inf")
    x[9] = torch.arange(classes, device="cuda") * 0.001
    x[10] = -torch.arange(classes, device="cuda") * 0.001
    x[11] = 3.0
    x[12, 5:] = float("nan")
    return x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,classes", [(4097, 2049), (4099, 3001), (5003, 1025), (4096, 5000)])
def test_long_rows_by_waves(rows, classes, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + classes)
    x = special(3 * torch.randn(rows, classes, generator=g, device="cuda"), g).to(dtype)
    t = torch.randint(-1, classes + 1, (rows,), generator=g, device="cuda")
    for top, ld, off in ((0, None, 0), (1, None, 0), (5, classes + 3, 1), (8, classes + 8, 0), (16, None, 0)):
        check(x, t, top, dtype, ld, off)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [8192 * 64, 8192 * 64 + 1, 8192 * 64 - 5])
def test_long_rows_by_waves_at_their_limit(classes, dtype):
    """The most classes that a wave takes, and what goes to workgroups: one row for all, the best ones among the last places."""
    g = torch.Generator(device="cuda").manual_seed(classes)
    one = torch.randn(1, classes, generator=g, device="cuda").to(dtype)
    one[0, -300:] = (5 + 0.125 * torch.arange(300, device="cuda").remainder(40)).to(dtype)
    got = head.log_probs(one.expand(4096, classes), torch.full((4096,), classes - 1, device="cuda"), top=16)
    lp = torch.log_softmax(one.double(), 1)
    ids = torch.sort(one, dim=1, descending=True, stable=True).indices[:, :16]
    assert torch.equal(got["top_ids"].long(), ids.expand(4096, 16))
    e = u * (144 + classes / 64) * (1 + math.log(classes) + 4 * 10)
    close(got["lse"], torch.logsumexp(one.double(), 1).cpu().expand(4096), e, F32, "lse")
    close(got["logp"], lp[:, -1].cpu().expand(4096), e, F32, "logp")
    close(got["top_logp"], lp.gather(1, ids).cpu().expand(4096, 16), e, F32, "top_logp")
    close(got["entropy"], -(lp.exp() * lp).sum(1).cpu().expand(4096), e, F32, "entropy")


@pytest.mark.parametrize("dtype,rows,classes", [(F32, 2_100_001, 7), (BF16, 2_100_001, 13), (F32, 65_601, 520), (F16, 65_601, 1030)])
def test_short_rows_take_several_turns(dtype, rows, classes):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (3 * torch.randn(rows, classes, generator=g, device="cuda")).to(dtype)
    x[5::9] = torch.randint(-2, 3, x[5::9].shape, generator=g, device="cuda").to(dtype)
    x[rows - 2] = -float("inf")
    check(x, torch.randint(-1, classes, (rows,), generator=g, device="cuda"), 3, dtype)
