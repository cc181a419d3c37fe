"""The operators record nothing for autograd: a tensor whose gradient is being recorded is refused, not detached without a word."""
import pytest
import torch

from paper_2309_11071_amd import head

pytestmark = pytest.mark.gpu


def test_recorded_tensors_are_refused():
    x, w, v = torch.ones(4, 8, device="cuda"), torch.ones(8, 3, device="cuda"), torch.ones(8, device="cuda")
    s = torch.ones(4, device="cuda")
    X, W, V, Q = (t.clone().requires_grad_() for t in (x, w, v, s))
    calls = [lambda: head.layer_norm(X), lambda: head.layer_norm(x, V), lambda: head.layer_norm(x, v, V), lambda: head.linear(X, w), lambda: head.linear(x, W),
             lambda: head.linear(x, w, W[0]), lambda: head.linear(x, w, residual=X[:, :3]), lambda: head.log_probs(X), lambda: head.log_probs_backward(X, None, s, g_logp=s),
             lambda: head.log_probs_backward(x, None, s, g_logp=Q), lambda: head.linear_backward(X[:, :3], x, w), lambda: head.linear_backward(x[:, :3], x, W),
             lambda: head.layer_norm_backward(x, X, s, s), lambda: head.layer_norm_backward(x, x, Q, s)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="autograd"):
            call()
            pytest.fail("call %d" % i)
        with torch.no_grad():
            call()
    assert torch.equal(head.linear(X.detach(), W.detach()), head.linear(x, w))
