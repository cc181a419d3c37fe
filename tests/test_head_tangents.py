"""Tensors with a tangent of forward mode: the operators would drop it without a word, so they raise."""
import pytest
import torch
from torch.autograd import forward_ad as fw

from paper_2309_11071_amd import head

F32 = torch.float32


def dual(t):
    return fw.make_dual(t, torch.ones_like(t))


def test_a_vector_with_a_tangent_raises():
    """On the CPU: the check itself, outside a level, for tensors without a tangent, detached ones and where forward mode is off."""
    t = torch.ones(3)
    assert head._vector(t, "t", 3, t, (F32,)) is t
    with fw.dual_level():
        d = dual(t)
        assert head._vector(t, "t", 3, t, (F32,)) is t
        for place in (torch.no_grad, torch.enable_grad):
            with place(), pytest.raises(ValueError, match="tangent"):
                head._vector(d, "t", 3, t, (F32,))
        head._vector(d.detach(), "t", 3, t, (F32,))
        with fw._set_fwd_grad_enabled(False):
            head._vector(d, "t", 3, t, (F32,))
        for other in (torch.zeros(3, dtype=torch.int64), torch.zeros(3, dtype=torch.uint8).view(head.E4M3)):
            head._vector(other, "t", 3, t, (other.dtype,))
    wanted = t.clone().requires_grad_()
    with pytest.raises(ValueError, match="requires a gradient"):
        head._vector(wanted, "t", 3, t, (F32,))


@pytest.mark.gpu
def test_every_operator_raises():
    x, w, v, s = (torch.randn(*n, device="cuda") for n in ((6, 8), (8, 5), (8,), (6,)))
    p, g = [torch.zeros(8, device="cuda")], [torch.ones(8, device="cuda")]
    mom, copy, factor = head.adamw_moments(p), [torch.zeros(8, dtype=torch.bfloat16, device="cuda")], torch.ones(1, device="cuda")
    labels = torch.zeros(6, dtype=torch.int64, device="cuda")
    calls = [
        (lambda x, v: head.layer_norm(x, v), (x, v)), (lambda x, v, r: head.rms_norm(x, v, residual=r), (x, v, x.clone())),
        (lambda d, x, r, v, t: head.rms_norm_backward(d, x, r, v, d_total=t), (x, x.clone(), s, v, x.clone())), (lambda x, a, b: head.gated(x, a, b), (x, w, w.clone())),
        (lambda d, x, a, b: head.gated_backward(d, x, a, b), (x[:, :5], x, w, w.clone())), (lambda x, a: head.linear(x, a), (x, w)),
        (lambda x: head.log_probs(x, labels, top=2), (x,)),
        (lambda p, g, m, c, f: head.adamw([p], [g], [(m, mom[0][1])], 1, copies=[c], grad_scale=f), (p[0], g[0], mom[0][0], copy[0], factor)),
    ]
    with fw.dual_level():
        for call, args in calls:
            call(*args)                                           # without a tangent as outside of a level
            for i in range(len(args)):
                with pytest.raises(ValueError, match="tangent"):
                    call(*args[:i], dual(args[i].clone()), *args[i + 1:])
                call(*args[:i], dual(args[i]).detach(), *args[i + 1:])
    for call, args in calls:
        call(*args)
