"""Tensors of an AdamW step that overlap, at the C boundary and in the binding's check: no launch happens, so no GPU is needed."""
import itertools

import pytest

from paper_2309_11071_amd import head
from test_block_arguments import C, E_ARG, Tensor, lib  # noqa: F401

M = 1 << 30          # addresses that nothing reads
N = 300
BYTES = dict(param=4 * N, grad=2 * N, copy=2 * N, m=N, v=N, m_scale=4 * 3, v_scale=4 * 3)      # 32-bit parameters, 16-bit gradients and copies, 8-bit moments
FIELDS = list(BYTES)


def step(lib, *tensors, **k):  # noqa: F811
    table = (Tensor * len(tensors))(*[Tensor(n=N, id=i, **t) for i, t in enumerate(tensors)])
    a = dict(tensors=C.addressof(table), count=len(tensors), pt=0, gt=1, ct=1, bits=8, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.01, step=1, step_at=None, gs=1.0, gs_at=None,
             seed=1, stream=None)
    return lib.ink_adamw(*{**a, **k}.values())


def places(tensors):
    """Tensors one behind the other, 4096 bytes apart."""
    return [{f: M + 4096 * (len(FIELDS) * i + j) for j, f in enumerate(FIELDS)} for i in range(tensors)]


# every pair of what a step changes, and every gradient with it, in one tensor and in two; by one element at either end, or one inside the other
@pytest.mark.parametrize("one,other", [p for p in itertools.product(FIELDS, FIELDS) if p != ("grad", "grad")])
def test_overlaps_are_refused(lib, one, other):  # noqa: F811
    for i, j in ((0, 0), (0, 1), (33, 2)):                        # (33: in another launch)
        if i == j and one == other:
            continue
        t = places(max(i, j) + 1)
        for at in (t[i][one] + BYTES[one] - 4, t[i][one] - BYTES[other] + 4, t[i][one] + 4, t[i][one]):
            t[j][other] = at
            assert step(lib, *t) == E_ARG, at - t[i][one]
            assert "memory that the step changes" in lib.ink_last_error(None).decode()


def test_step_and_scale_in_memory_that_changes(lib):  # noqa: F811
    t = places(1)
    for k in (dict(step_at=t[0]["param"] + 8), dict(step_at=t[0]["v_scale"] - 0), dict(gs_at=t[0]["m"] + 4), dict(gs_at=t[0]["m_scale"] + 8)):
        assert step(lib, *t, **k) == E_ARG and "step_at or grad_scale_at stands" in lib.ink_last_error(None).decode()


def test_the_bindings_check():
    head._apart([], [])
    head._apart([(0, 8), (8, 12), (20, 24)], [(12, 20), (12, 14), (13, 20), (24, 30)])
    for changed in ([(0, 8), (7, 12)], [(7, 12), (0, 8)], [(0, 8), (0, 8)], [(0, 100), (50, 60)], [(50, 60), (0, 100), (200, 201)]):
        with pytest.raises(ValueError):
            head._apart(changed, [])
    for read in ((0, 1), (7, 9), (11, 13), (19, 21), (0, 30), (10, 22), (21, 22)):
        with pytest.raises(ValueError):
            head._apart([(0, 8), (8, 12), (20, 24)], [(13, 14), read])
