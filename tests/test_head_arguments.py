"""Argument checks of an answer head's operators at the C boundary: no launch happens, so no GPU is needed."""
import ctypes as C
import os

import pytest

from paper_2309_11071_amd import binding

E_ARG = 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.lib_path()):
        pytest.skip("libink.so not built")
    from paper_2309_11071_amd import head
    return head._functions()


M = 1 << 20          # an address that nothing reads


def norm(lib, **k):
    a = dict(x=M, ld_x=8, weight=M, bias=M, rows=4, cols=8, type=0, param=0, eps=1e-5, y=M, ld_y=8, mean=M, rstd=M, stream=None)
    return lib.ink_layer_norm(*{**a, **k}.values())


def norm_grad(lib, **k):
    a = dict(dy=M, ld_dy=8, x=M, ld_x=8, mean=M, rstd=M, weight=M, rows=4, cols=8, type=0, param=0, dx=M, ld_dx=8, dw=M, db=M, work=M, n=1 << 20, stream=None)
    return lib.ink_layer_norm_backward(*{**a, **k}.values())


def linear(lib, **k):
    a = dict(x=M, ld_x=8, w=M, ld_w=5, bias=M, res=M, ld_res=5, rows=4, cols=8, out=5, type=1, out_type=1, act=0, y=M, ld_y=5, pre=M, ld_pre=5, stream=None)
    return lib.ink_linear(*{**a, **k}.values())


def linear_grad(lib, **k):
    a = dict(dy=M, ld_dy=5, x=M, ld_x=8, w=M, ld_w=5, pre=M, ld_pre=5, rows=4, cols=8, out=5, type=1, dy_type=1, act=2, dx=M, ld_dx=8, dw=M, ld_dw=5, db=M,
             work=M, n=1 << 30, stream=None)
    return lib.ink_linear_backward(*{**a, **k}.values())


def probs(lib, **k):
    a = dict(z=M, ld=5, t=M, tb=8, rows=4, classes=5, type=0, scale=1.0, top=2, logp=M, ent=M, lse=M, ids=M, top_logp=M, work=M, n=1 << 30, stream=None)
    return lib.ink_log_probs(*{**a, **k}.values())


def probs_grad(lib, **k):
    a = dict(z=M, ld=5, t=M, tb=8, lse=M, ent=M, g=M, h=M, rows=4, classes=5, type=0, scale=1.0, out=M, ld_out=5, stream=None)
    return lib.ink_log_probs_backward(*{**a, **k}.values())


BAD = [
    (norm, dict(type=3)), (norm, dict(type=-1)), (norm, dict(param=1)), (norm, dict(rows=-1)), (norm, dict(rows=1 << 31)), (norm, dict(cols=0)),
    (norm, dict(cols=16385)), (norm, dict(eps=0.0)), (norm, dict(eps=-1.0)), (norm, dict(eps=float("nan"))), (norm, dict(eps=float("inf"))),
    (norm, dict(x=None)), (norm, dict(x=M + 2)), (norm, dict(ld_x=7)), (norm, dict(ld_x=-8)), (norm, dict(y=None)), (norm, dict(ld_y=7)), (norm, dict(ld_y=0)),
    (norm, dict(weight=M + 1)), (norm, dict(bias=M + 2)), (norm, dict(mean=M + 1)), (norm, dict(rstd=M + 2)),
    (norm_grad, dict(type=9)), (norm_grad, dict(dy=None)), (norm_grad, dict(x=None)), (norm_grad, dict(mean=None)), (norm_grad, dict(rstd=None)),
    (norm_grad, dict(dx=M + 1)), (norm_grad, dict(ld_dx=0)), (norm_grad, dict(work=None)), (norm_grad, dict(n=8)), (norm_grad, dict(work=M + 2)),
    (norm_grad, dict(db=M + 2)), (norm_grad, dict(dw=M + 1)),
    (linear, dict(type=4)), (linear, dict(out_type=2)), (linear, dict(act=4)), (linear, dict(act=-1)), (linear, dict(cols=0)), (linear, dict(out=0)),
    (linear, dict(out=20000)), (linear, dict(rows=-5)), (linear, dict(x=None)), (linear, dict(w=None)), (linear, dict(ld_w=4)), (linear, dict(y=None)),
    (linear, dict(y=M + 1)), (linear, dict(ld_y=4)), (linear, dict(ld_res=4)), (linear, dict(ld_pre=4)), (linear, dict(ld_pre=0)), (linear, dict(bias=M + 1)),
    (linear_grad, dict(dy=None)), (linear_grad, dict(pre=None)), (linear_grad, dict(x=None)), (linear_grad, dict(w=None)), (linear_grad, dict(ld_dx=0)),
    (linear_grad, dict(ld_dw=4)), (linear_grad, dict(work=None)), (linear_grad, dict(n=16)), (linear_grad, dict(work=M + 4)), (linear_grad, dict(db=M + 1)),
    (linear_grad, dict(type=2, dy_type=0)), (linear_grad, dict(type=0, dy_type=1)), (linear_grad, dict(act=7)),
    (probs, dict(type=3)), (probs, dict(classes=0)), (probs, dict(classes=(1 << 30) + 1)), (probs, dict(rows=-1)), (probs, dict(scale=0.0)),
    (probs, dict(scale=float("nan"))), (probs, dict(scale=float("inf"))), (probs, dict(top=6)), (probs, dict(top=-1)), (probs, dict(classes=40, ld=40, top=17)),
    (probs, dict(z=None)), (probs, dict(ld=4)), (probs, dict(tb=2)), (probs, dict(t=M + 4)), (probs, dict(logp=M + 1)), (probs, dict(ids=M + 2)),
    (probs, dict(classes=100_000, ld=100_000, work=None)), (probs, dict(classes=100_000, ld=100_000, n=10)),
    (probs_grad, dict(lse=None)), (probs_grad, dict(ent=None)), (probs_grad, dict(g=None, h=None)), (probs_grad, dict(out=None)), (probs_grad, dict(ld_out=4)),
    (probs_grad, dict(ld_out=0)), (probs_grad, dict(z=M + 2)), (probs_grad, dict(g=M + 1)), (probs_grad, dict(scale=-1.0)),
]


@pytest.mark.parametrize("i", range(len(BAD)))
def test_bad_arguments_are_refused(lib, i):
    call, change = BAD[i]
    assert call(lib, **change) == E_ARG
    name = {norm: "ink_layer_norm:", norm_grad: "ink_layer_norm_backward:", linear: "ink_linear:", linear_grad: "ink_linear_backward:",
            probs: "ink_log_probs:", probs_grad: "ink_log_probs_backward:"}[call]
    assert lib.ink_last_error(None).decode().startswith(name)


def test_no_rows_need_no_memory(lib):
    none = dict(rows=0)
    assert norm(lib, x=None, y=None, mean=None, rstd=None, **none) == 0
    assert norm_grad(lib, dy=None, x=None, mean=None, rstd=None, dx=None, dw=None, db=None, work=None, n=0, **none) == 0
    assert linear(lib, x=None, y=None, res=None, pre=None, **none) == 0
    assert linear_grad(lib, dy=None, x=None, pre=None, dx=None, dw=None, db=None, work=None, n=0, **none) == 0
    assert probs(lib, z=None, work=None, n=0, **none) == 0
    assert probs_grad(lib, z=None, lse=None, out=None, **none) == 0


def test_work_sizes(lib):
    assert lib.ink_layer_norm_backward_work(0, 8, 0) == 0 and lib.ink_layer_norm_backward_work(5, 8, 7) == 0
    assert lib.ink_layer_norm_backward_work(1, 8, 0) == 2 * 8 * 4
    assert lib.ink_linear_backward_work(0, 8, 8) == 0 and lib.ink_linear_backward_work(1, 8, 5) >= 9 * 5 * 4
    assert lib.ink_log_probs_work(4, 100, 0, 5) == 0 and lib.ink_log_probs_work(4, 100_000, 0, 5) > 0
    for rows in (1, 1000, (1 << 31) - 1):        # the largest problems do not wrap around
        for cols in (1, 602, 16384):
            assert 0 < lib.ink_layer_norm_backward_work(rows, cols, 1) < 1 << 31
            assert lib.ink_linear_backward_work(rows, cols, 16384) >= (cols + 1) * 16384 * 4


def test_functions_have_the_headers_argument_lists(lib):
    """One ctypes argument for each parameter that include/ink.h declares, of its width."""
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "ink.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    kinds = {"int32_t": C.c_int32, "int64_t": C.c_int64, "size_t": C.c_size_t, "float": C.c_float}
    seen = 0
    for name in ("ink_layer_norm", "ink_layer_norm_backward", "ink_linear", "ink_linear_backward", "ink_log_probs", "ink_log_probs_backward",
                 "ink_layer_norm_backward_work", "ink_linear_backward_work", "ink_log_probs_work"):
        args = re.search(r"\b%s\s*\(([^)]*)\)\s*;" % name, text).group(1).split(",")
        want = [C.c_void_p if "*" in a else kinds[a.split()[0]] for a in args]
        assert tuple(want) == tuple(getattr(lib, name).argtypes), name
        seen += 1
    assert seen == 9
