"""The operators of a head of residual blocks together, as the example uses them."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from paper_2309_11071_amd import head

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("residual_head", os.path.join(ROOT, "examples", "residual_head.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain(params, rows, labels, blocks):
    """The head's loss in 64 bits on the CPU, with autograd."""
    def norm(x, w):
        return x * (x.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w
    x = rows
    for b in range(blocks):
        gamma, gate, up, down = params[4 * b:4 * b + 4]
        y = norm(x, gamma)
        x = x + (torch.nn.functional.silu(y @ gate) * (y @ up)) @ down
    logits = norm(x, params[-3]) @ params[-2] + params[-1]
    logp = torch.log_softmax(logits, 1)
    known = labels >= 0
    return -logp[known].gather(1, labels[known][:, None]).sum() / known.sum()


@pytest.mark.parametrize("kind,rows,dim,hidden", [("f32", 70, 24, 64), ("f32", 300, 64, 171), ("bf16", 300, 64, 171), ("f16", 300, 64, 171), ("bf16", 5, 40, 100),
                                                  ("bf16", 33000, 64, 100)])
def test_gradients_of_the_whole_head(example, kind, rows, dim, hidden):
    """Against autograd of the formulas in 64 bits, relative in the 2-norm.  A value passes some 6 operators a block and 4 at the end, forwards and back: 32 for
    two blocks.  In 32 bits each errs by at most the longest sum (512 terms of hidden, dim or rows in a chain) times 2^-24, in 16 bits by its rounding, whose
    root mean square is 2^-9 / sqrt 3 (bfloat16) or 2^-12 / sqrt 3; independent errors add as squares, and a factor of 4 covers how far normalised rows and
    products of two factors pass them on."""
    g = torch.Generator().manual_seed(rows)
    dtype = dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)[kind]
    model = example.ResidualHead(dim, hidden, 2, 9, dtype, seed=rows)
    model.params = [(p + 0.1 * torch.randn(p.shape, generator=g).cuda()).to(dtype).float() if p.dim() == 1 else p.to(dtype).float() for p in model.params]
    if model.copies is not None:
        model.copies = [p.to(dtype) for p in model.params]
    x = torch.randn(rows, dim, generator=g).to(dtype)
    labels = torch.randint(-1, 9, (rows,), generator=g)
    logits, kept = model.forward(x.cuda())
    out = head.log_probs(logits, labels.cuda())
    n = int((labels >= 0).sum())
    scale = 1024.0 if kind == "f16" else 1.0
    d = head.log_probs_backward(logits, labels.cuda(), out["lse"], g_logp=torch.full((rows,), -scale / n, device="cuda"))
    grads, d_rows = model.backward(d, kept)
    params = [p.double().cpu().requires_grad_() for p in model.params]
    wide = x.double().requires_grad_()
    loss = plain(params, wide, labels, 2)
    loss.backward()
    loss = loss.detach()
    tol = {"f32": 4 * 32 * 512 * 2.0 ** -24, "bf16": 4 * (32 / 3) ** 0.5 * 2.0 ** -9, "f16": 4 * (32 / 3) ** 0.5 * 2.0 ** -12}[kind]
    assert abs(float(-out["logp"].sum() / n) - float(loss)) <= tol * max(1.0, float(loss))
    for i, (got, p) in enumerate(zip(grads + [d_rows], params + [wide])):
        want = p.grad
        assert float((got.double().cpu() / scale - want).norm()) <= tol * float(want.norm()), (i, float((got.double().cpu() / scale - want).norm() / want.norm()))


def test_a_step_of_training_in_a_graph(example):
    """Forward, backward and AdamW captured once, replayed with eager work between, against the same steps called eagerly."""
    g = torch.Generator().manual_seed(2)
    x, labels = torch.randn(500, 32, generator=g).cuda(), torch.randint(-1, 5, (500,), generator=g).cuda()
    models = [example.ResidualHead(32, 85, 1, 5, torch.bfloat16, bits=8, seed=3) for _ in range(2)]
    grad = torch.full((500,), -1 / 500, device="cuda")
    at = torch.zeros((), dtype=torch.int64, device="cuda")

    def step(m, t):
        logits, kept = m.forward(x)
        out = head.log_probs(logits, labels)
        grads, _ = m.backward(head.log_probs_backward(logits, labels, out["lse"], g_logp=grad), kept)
        head.adamw(m.params, grads, m.moments, t, copies=m.copies, seed=7)
    held = [t for t in models[0].params + models[0].copies + [x for e in models[0].moments for x in e]]
    was = [t.clone() for t in held]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(models[0], at)
        for t, w in zip(held, was):
            t.copy_(w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        at.add_(1)
        step(models[0], at)
    for t in (1, 2, 3):
        graph.replay()
        torch.cuda.synchronize()
        step(models[1], t)
        other = [w for w in models[1].params + models[1].copies + [x for e in models[1].moments for x in e]]
        for u, v in zip(held, other):
            assert torch.equal(u.view(torch.uint8), v.view(torch.uint8)), t


@pytest.mark.parametrize("kind,bits", [("bf16", 8), ("f16", 8), ("f32", 32)])
def test_the_example_runs(example, kind, bits):
    losses, kept, whole = example.main(["--steps", "20", "--batches", "2", "--type", kind, "--bits", str(bits)])
    assert np.isfinite(losses).all()
    # rows are normalised, rounded to 8 bits and multiplied one by one, in whichever launch: the kernels of few and of many rows may round differently,
    # which can swap classes whose logits agree to the last bits only
    assert float((kept == whole).all(1).float().mean()) > 0.99
