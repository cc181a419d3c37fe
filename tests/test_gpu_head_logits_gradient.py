"""The gradient of log probabilities where lse is so large that 32 bits do not hold log p beside it."""
import math

import pytest
import torch

from paper_2309_11071_amd import head
from test_gpu_head import TYPES, close, gen, table, u
from test_gpu_head_logits import SHAPES, exact, far_rows

pytestmark = pytest.mark.gpu


def gradient(x, t, gl, ge, scale):
    """The gradient in 64 bits from the logits alone, and its bound."""
    lse, lp, ent, e = exact(x, scale)
    p = lp.exp()
    gl, ge = gl.double()[:, None], ge.double()[:, None]
    has = (t >= 0)[:, None].double()
    one = torch.zeros_like(p).scatter_(1, t.clamp(min=0)[:, None], has)
    flat = torch.where(p > 0, p * (lp + ent[:, None]), torch.zeros_like(p))
    want = scale * (gl * (one - has * p) - ge * flat)
    e_lp = e[:, None] + 8 * u * (1 + lp.clamp(min=-1e3).abs())
    size = p * (gl.abs() + ge.abs() * (lp.clamp(min=-1e3).abs() + ent[:, None]))
    return want, scale * (size * (e_lp + 4 * u) + p * ge.abs() * (e_lp + 4 * e[:, None] + u * ent[:, None]) + 4 * u * gl.abs() * one)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,classes", SHAPES)
def test_gradient_far_from_zero(rows, classes, dtype):
    g = gen(rows * 3 + classes)
    x = far_rows(rows, classes, dtype, g)
    x[1] = (3 * torch.randn(classes, generator=g)).to(dtype)             # a row near zero among them
    t = torch.randint(-1, classes, (rows,), generator=g)
    gl, ge = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    for scale, ld, off, use in ((1.0, classes, 0, "both"), (0.5, classes + 3, 1, "logp"), (2.0, classes, 0, "both")):
        _, _, ent, _ = exact(x, scale)
        out = head.log_probs(x.cuda(), t.cuda(), scale=scale)
        got = head.log_probs_backward(table(x, ld, off), t.cuda(), out["lse"], ent.float().cuda(), g_logp=gl.cuda(),
                                      g_entropy=ge.cuda() if use == "both" else None, scale=scale)
        want, e = gradient(x, t, gl, ge if use == "both" else 0 * ge, scale)
        e[1] += e.new_tensor(4 * 32 * u) * scale                          # lse of that row, below 32, rounded
        close(got, want, e, dtype, "dlogits " + use)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,classes", [(5, 5), (20, 47), (9, 700), (6, 3000), (3, 70_001)])
def test_gradient_of_rows_at_the_ends_of_a_type(rows, classes, dtype):
    """A row that lowest values mask altogether is one of equal logits: p = 1 / C.  One that -inf masks has no gradient."""
    big = float(torch.finfo(dtype).max)
    x = torch.full((rows, classes), -big)
    x[1] = big
    x[2] = -float("inf")
    x[3::2, 3] = 1.0
    x = x.to(dtype)
    t = torch.full((rows,), 1)
    t[3::2] = 3
    gl, ge = torch.full((rows,), -0.75), torch.full((rows,), 0.5)
    for scale in (1.0, 2.0):
        out = head.log_probs(x.cuda(), t.cuda(), scale=scale)
        got = head.log_probs_backward(table(x), t.cuda(), out["lse"], out["entropy"], g_logp=gl.cuda(), g_entropy=ge.cuda(), scale=scale).double().cpu()
        one = torch.zeros(classes, dtype=torch.float64)
        one[1] = 1
        want = (-0.75 * scale * (one - 1.0 / classes)).expand(rows, classes)
        # p errs by its sum's chain; the entropy's part, p (log p + H), is zero but for the errors of log p and H
        tol = scale * u * (144 + classes / 64) * (1 + math.log(classes)) * 3 / classes
        equal = torch.arange(rows) % 2 == 0
        equal[1], equal[2] = True, False
        close(got[equal], want[equal], tol, dtype, "rows of equal logits")
        assert (got[~equal] == 0).all(), "one class left, or none"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [7, 300, 5003])
def test_large_gradients_of_masked_classes(dtype, classes):
    """p = 0 and log p = -inf: such a class takes no part in the entropy, whatever the entropy's gradient is."""
    x = torch.zeros(3, classes).to(dtype)
    x[:, 2:] = -float("inf")
    x[2] -= 1000
    out = head.log_probs(x.cuda(), None)
    h = torch.full((3,), 1e9).cuda()
    got = head.log_probs_backward(x.cuda(), None, out["lse"], out["entropy"], g_entropy=h).double().cpu()
    assert (got[:, 2:] == 0).all()
    # -h p (log p + H): zero but for the errors of log p, H and lse, each of a few u (lse of the third row is formed anew)
    assert got[:, :2].abs().max() <= 1e9 * 0.5 * 16 * u
