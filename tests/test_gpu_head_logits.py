"""Log probabilities of rows whose logits are far from zero: log p depends on differences of logits only, and so do its digits.

u = 2^-24.  With d = z - max z and S = sum e^d, log p_t = d_t - log S errs by a few u of d_t, and by what S errs by: u times the additions
of its longest chain, and a few u of sum p |d| from the exponents.  No bound here knows the size of the logits.
"""
import math

import pytest
import torch

from paper_2309_11071_amd import head
from test_gpu_head import F32, TYPES, close, gen, table, u

pytestmark = pytest.mark.gpu


def exact(x, scale):
    """lse, log p, entropy in 64 bits, and the bound of a log probability but for the rounding of d_t."""
    z = x.double() * scale
    d = z - z.amax(1, keepdim=True)
    s = d.exp().sum(1, keepdim=True)
    lp = d - s.log()
    p = lp.exp()
    flat = torch.where(p > 0, p * d, torch.zeros_like(p))
    e = u * (16 + 128 + x.shape[1] / 64) * (1 + math.log(x.shape[1] + 1) + flat.abs().sum(1))
    ent = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    return torch.logsumexp(z, 1), lp, ent, e


SHAPES = [(3, 2), (5, 7), (40, 9), (60, 47), (33, 172), (20, 300), (9, 1000), (5, 2048), (3, 2049), (4, 5003), (2, 70_001), (4100, 2060)]


def far_rows(rows, classes, dtype, g):
    """Rows around offsets of either sign, the largest such that the type's values there still differ."""
    off = torch.tensor([2.0e4, 1000.0, -3.0e4, -700.0, 5.0e3])[torch.arange(rows) % 5][:, None]
    x = off + (3 if dtype == F32 else 40) * torch.randn(rows, classes, generator=g)
    return x.to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,classes", SHAPES)
def test_log_p_keeps_its_digits_far_from_zero(rows, classes, dtype):
    g = gen(rows + classes)
    x = far_rows(rows, classes, dtype, g)
    t = torch.randint(0, classes, (rows,), generator=g)
    for scale, top, ld, off in ((1.0, min(5, classes), classes, 0), (0.5, 0, classes + 3, 1), (0.125, min(16, classes), classes, 0)):
        got = head.log_probs(table(x, ld, off), t.cuda(), top=top, scale=scale)
        lse, lp, ent, e = exact(x, scale)
        mine = lp.gather(1, t[:, None])
        close(got["logp"][:, None], mine, e[:, None] + 4 * u * mine.abs(), F32, "logp")
        best = torch.gather(lp, 1, got["top_ids"].cpu().long())
        close(got["top_logp"], best, e[:, None] + 4 * u * best.abs(), F32, "top_logp")
        close(got["entropy"], ent, 4 * e, F32, "entropy")
        close(got["lse"], lse, e + 2 * u * lse.abs(), F32, "lse")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,classes", [(5, 5), (20, 47), (9, 700), (6, 3000), (3, 70_001), (4100, 2060)])
def test_rows_at_the_ends_of_a_type(rows, classes, dtype):
    """Every class at the type's lowest value, or its largest, or all but one: finite logits, of which scale * logit may be none."""
    big = float(torch.finfo(dtype).max)
    x = torch.full((rows, classes), -big)
    x[1] = big
    x[2::2, 3] = 1.0
    x = x.to(dtype)
    t = torch.full((rows,), 1)
    t[2] = 3
    for scale in (1.0, 2.0, 64.0):
        got = {k: v.cpu() for k, v in head.log_probs(table(x), t.cuda(), top=2, scale=scale).items()}
        even = math.log(classes)
        tol = u * (144 + classes / 64) * (1 + even)
        for r in (0, 1):
            assert abs(float(got["logp"][r]) + even) <= tol and abs(float(got["entropy"][r]) - even) <= tol
            assert (got["top_logp"][r] + even).abs().max() <= tol and got["top_ids"][r].tolist() == [0, 1]
            want = (2 * r - 1) * big * scale             # + log C, far below its last digit
            assert math.isfinite(float(got["lse"][r])), "only a row of masked classes has -inf"
            assert abs(float(got["lse"][r]) - max(-3.4028234e38, min(3.4028234e38, want))) <= abs(want) * 1e-6 + even
        assert float(got["logp"][2]) == 0 and float(got["entropy"][2]) == 0 and float(got["lse"][2]) == scale
        assert got["top_ids"][2].tolist() == [3, 0] and float(got["top_logp"][2, 0]) == 0
        assert float(got["logp"][4 if rows > 4 else 2]) == (float(torch.tensor((-big - 1) * scale, dtype=torch.float64).float()) if rows > 4 else 0)
