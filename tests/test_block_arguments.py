"""Argument checks of the residual blocks' operators and of the AdamW step at the C boundary: no launch happens, so no GPU is needed."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2309_11071_amd import binding, head

E_ARG = 1
M = 1 << 20          # an address that nothing reads
MAX_COLS, MAX_ROWS = 16384, (1 << 31) - 1
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Tensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("param", "grad", "copy", "m", "v", "m_scale", "v_scale")] + [("n", C.c_int64), ("id", C.c_int64)]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.lib_path()):
        pytest.skip("libink.so not built")
    return head._functions()


def rms(lib, **k):
    a = dict(x=M, ld_x=8, res=M, ld_res=8, weight=M, rows=4, cols=8, type=1, param=1, eps=1e-6, out=1, y=M, ld_y=8, scale=None, total=M, ld_total=8, rstd=M,
             stream=None)
    return lib.ink_rms_norm(*{**a, **k}.values())


def rms_grad(lib, **k):
    a = dict(dy=M, ld_dy=8, total=M, ld_total=8, rstd=M, weight=M, dt=M, ld_dt=8, rows=4, cols=8, type=0, param=0, dx=M, ld_dx=8, dw=M, work=M, n=1 << 20, stream=None)
    return lib.ink_rms_norm_backward(*{**a, **k}.values())


def gated(lib, **k):
    a = dict(x=M, ld_x=8, xs=None, wg=M, ld_g=5, wu=M, ld_u=5, gs=None, us=None, rows=4, cols=8, hidden=5, type=1, out=1, act=3, h=M, ld_h=5, stream=None)
    return lib.ink_gated(*{**a, **k}.values())


def gated_8(lib, **k):
    return gated(lib, **{**dict(type=3, ld_g=8, ld_u=8, xs=M, gs=M, us=M), **k})


def gated_grad(lib, **k):
    a = dict(dh=M, ld_dh=5, x=M, ld_x=8, wg=M, ld_g=5, wu=M, ld_u=5, rows=4, cols=8, hidden=5, type=1, act=2, dx=M, ld_dx=8, dg=M, ld_dg=5, du=M, ld_du=5, work=M,
             n=1 << 30, stream=None)
    return lib.ink_gated_backward(*{**a, **k}.values())


def adamw(lib, **k):
    t = {**dict(param=M, grad=M, copy=M, m=M, v=M, m_scale=M, v_scale=M, n=100, id=0), **{f: k.pop(f) for f in list(k) if f in dict(Tensor._fields_)}}
    table = (Tensor * 2)(Tensor(n=0), Tensor(**t))
    a = dict(tensors=C.addressof(table), count=2, pt=0, gt=1, ct=1, bits=8, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.01, step=1, step_at=None, gs=1.0, gs_at=None, seed=1,
             stream=None)
    return lib.ink_adamw(*{**a, **k}.values())


NAN, INF = float("nan"), float("inf")
BAD = [
    (rms, dict(type=3)), (rms, dict(type=-1)), (rms, dict(param=2)), (rms, dict(rows=-1)), (rms, dict(rows=MAX_ROWS + 1)), (rms, dict(cols=0)),
    (rms, dict(cols=MAX_COLS + 1)), (rms, dict(eps=0.0)), (rms, dict(eps=NAN)), (rms, dict(eps=INF)), (rms, dict(out=0)), (rms, dict(out=2)), (rms, dict(out=4)),
    (rms, dict(x=None)), (rms, dict(x=M + 1)), (rms, dict(ld_x=7)), (rms, dict(ld_x=-8)), (rms, dict(res=M + 1)), (rms, dict(ld_res=7)), (rms, dict(total=None)),
    (rms, dict(total=M + 1)), (rms, dict(ld_total=7)), (rms, dict(ld_total=0)), (rms, dict(y=None)), (rms, dict(ld_y=0)), (rms, dict(y=M + 1)), (rms, dict(weight=M + 1)),
    (rms, dict(rstd=M + 2)), (rms, dict(out=3, scale=None)), (rms, dict(out=3, scale=M + 2)),
    (rms_grad, dict(type=3)), (rms_grad, dict(param=1)), (rms_grad, dict(dy=None)), (rms_grad, dict(total=None)), (rms_grad, dict(rstd=None)), (rms_grad, dict(rstd=M + 1)),
    (rms_grad, dict(ld_dt=7)), (rms_grad, dict(dt=M + 2)), (rms_grad, dict(dx=M + 1)), (rms_grad, dict(ld_dx=0)), (rms_grad, dict(dw=M + 2)), (rms_grad, dict(work=None)),
    (rms_grad, dict(work=M + 4)), (rms_grad, dict(n=31)),
    (gated, dict(type=4)), (gated, dict(type=-1)), (gated, dict(out=0)), (gated, dict(act=4)), (gated, dict(act=-1)), (gated, dict(rows=-1)), (gated, dict(cols=0)),
    (gated, dict(hidden=0)), (gated, dict(cols=MAX_COLS + 1)), (gated, dict(hidden=MAX_COLS + 1)), (gated, dict(x=None)), (gated, dict(x=M + 1)), (gated, dict(wg=None)),
    (gated, dict(wu=None)), (gated, dict(ld_g=4)), (gated, dict(ld_u=4)), (gated, dict(h=None)), (gated, dict(ld_h=4)), (gated, dict(ld_h=0)),
    (gated_8, dict(out=3)), (gated_8, dict(out=5)), (gated_8, dict(ld_g=7)), (gated_8, dict(ld_u=7)), (gated_8, dict(xs=None)), (gated_8, dict(gs=None)), (gated_8, dict(us=None)),
    (gated_8, dict(xs=M + 2)), (gated_8, dict(gs=M + 1)), (gated_8, dict(us=M + 3)), (gated_8, dict(h=M + 1)),
    (gated_grad, dict(type=3)), (gated_grad, dict(act=4)), (gated_grad, dict(rows=-1)), (gated_grad, dict(dh=None)), (gated_grad, dict(x=None)), (gated_grad, dict(wg=None)),
    (gated_grad, dict(wu=M + 1)), (gated_grad, dict(ld_dx=7)), (gated_grad, dict(ld_dg=4)), (gated_grad, dict(ld_du=0)), (gated_grad, dict(dg=M + 1)), (gated_grad, dict(du=M + 1)),
    (gated_grad, dict(work=None)), (gated_grad, dict(work=M + 8)), (gated_grad, dict(n=100)),
    (adamw, dict(count=-1)), (adamw, dict(tensors=None)), (adamw, dict(pt=2)), (adamw, dict(pt=3)), (adamw, dict(gt=3)), (adamw, dict(ct=0)), (adamw, dict(ct=3)),
    (adamw, dict(pt=1, ct=1)), (adamw, dict(bits=16)), (adamw, dict(lr=-1.0)), (adamw, dict(lr=NAN)), (adamw, dict(lr=INF)), (adamw, dict(b1=1.0)), (adamw, dict(b1=-0.1)),
    (adamw, dict(b2=1.0)), (adamw, dict(b2=NAN)), (adamw, dict(eps=0.0)), (adamw, dict(eps=1e-40)), (adamw, dict(eps=INF)), (adamw, dict(wd=-1.0)), (adamw, dict(wd=INF)),
    (adamw, dict(gs=INF)), (adamw, dict(gs=NAN)), (adamw, dict(step=0)), (adamw, dict(step_at=M + 4)), (adamw, dict(gs_at=M + 2)),
    (adamw, dict(n=-1)), (adamw, dict(n=1 << 40)), (adamw, dict(param=None)), (adamw, dict(grad=None)), (adamw, dict(copy=None)), (adamw, dict(m=None)), (adamw, dict(v=None)),
    (adamw, dict(m_scale=None)), (adamw, dict(v_scale=M + 2)), (adamw, dict(param=M + 2)), (adamw, dict(grad=M + 1)), (adamw, dict(copy=M + 1)), (adamw, dict(bits=32, m=M + 1)),
]
NAMES = {rms: "ink_rms_norm:", rms_grad: "ink_rms_norm_backward:", gated: "ink_gated:", gated_8: "ink_gated:", gated_grad: "ink_gated_backward:", adamw: "ink_adamw:"}


@pytest.mark.parametrize("i", range(len(BAD)))
def test_bad_arguments_are_refused(lib, i):
    call, change = BAD[i]
    assert call(lib, **change) == E_ARG
    assert lib.ink_last_error(None).decode().startswith(NAMES[call])


def test_rates_that_pass_a_floats_range_are_refused(lib):
    """lr / (1 - beta1) and lr times the decay are floats on the device: their factors end at 1e18."""
    assert adamw(lib, lr=1.1e18) == E_ARG and adamw(lib, wd=1.1e18) == E_ARG
    assert adamw(lib, n=0, lr=1e18, wd=1e18) == 0


def test_no_rows_need_no_memory(lib):
    assert rms(lib, x=None, res=None, y=None, total=None, rstd=None, rows=0) == 0
    assert rms(lib, x=None, res=M, y=None, total=None, rstd=None, rows=0, out=3) == 0
    assert rms_grad(lib, dy=None, total=None, rstd=None, dt=None, dx=None, dw=None, work=None, n=0, rows=0) == 0
    assert gated(lib, x=None, h=None, rows=0) == 0 and gated_8(lib, x=None, xs=None, h=None, rows=0) == 0
    assert gated_grad(lib, dh=None, x=None, dx=None, dg=None, du=None, work=None, n=0, rows=0) == 0
    assert adamw(lib, tensors=None, count=0) == 0 and adamw(lib, n=0, param=None, grad=None) == 0


def test_the_ends_of_the_ranges(lib):
    assert rms(lib, rows=0, cols=MAX_COLS, ld_x=MAX_COLS) == 0
    assert gated(lib, rows=0, cols=MAX_COLS, hidden=MAX_COLS, ld_g=MAX_COLS, ld_u=MAX_COLS) == 0
    assert adamw(lib, n=0, lr=0.0, b1=0.0, b2=0.0, wd=0.0, step=1 << 62) == 0
    for rows in (1, 1000, MAX_ROWS):
        for cols in (1, 602, MAX_COLS):
            assert 0 < lib.ink_rms_norm_backward_work(rows, cols, 1) < 1 << 31
            for type in (0, 1, 2):
                assert lib.ink_gated_backward_work(rows, cols, 1, type) > 0
                # dg and du of a part of the rows, and partial matrices: as much for any number of rows
                assert 0 < lib.ink_gated_backward_work(rows, cols, MAX_COLS, type) < (2200 << 20) + cols * MAX_COLS * 16
    assert lib.ink_gated_backward_work(0, 8, 8, 0) == lib.ink_gated_backward_work(4, 8, 8, 3) == lib.ink_gated_backward_work(4, 0, 8, 0) == 0
    assert lib.ink_gated_backward_work(4, 8, MAX_COLS + 1, 0) == lib.ink_rms_norm_backward_work(4, MAX_COLS + 1, 0) == lib.ink_rms_norm_backward_work(4, 8, 3) == 0


def test_functions_have_the_headers_argument_lists(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ink.h")).read(), flags=re.S)
    kinds = {"int32_t": C.c_int32, "int64_t": C.c_int64, "size_t": C.c_size_t, "float": C.c_float, "double": C.c_double, "uint64_t": C.c_uint64}
    for name in ("ink_rms_norm", "ink_rms_norm_backward", "ink_gated", "ink_gated_backward", "ink_adamw", "ink_rms_norm_backward_work", "ink_gated_backward_work"):
        args = re.search(r"\b%s\s*\(([^)]*)\)\s*;" % name, text).group(1).split(",")
        want = [C.c_void_p if "*" in a else kinds[a.split()[0]] for a in args]
        assert tuple(want) == tuple(getattr(lib, name).argtypes), name


def test_the_tensor_struct_is_the_headers():
    import subprocess
    import tempfile
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "ink.h"\nint main(void) { printf("%zu %zu %zu %zu %d %d\\n", sizeof(ink_adamw_tensor), ' \
          'offsetof(ink_adamw_tensor, m), offsetof(ink_adamw_tensor, n), offsetof(ink_adamw_tensor, id), INK_ADAMW_BLOCK, INK_E4M3); return 0; }\n'
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "t.c"), "w").write(src)
        subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", os.path.join(d, "t"), os.path.join(d, "t.c")])
        got = [int(x) for x in subprocess.check_output([os.path.join(d, "t")]).split()]
    assert got == [C.sizeof(Tensor), Tensor.m.offset, Tensor.n.offset, Tensor.id.offset, head.ADAMW_BLOCK, head._TYPES_8[head.E4M3]]


# ------------------------------------------------------------------------------------ the binding
def test_the_binding_refuses_tensors_that_are_not_on_a_gpu():
    x, w = torch.zeros(4, 8), torch.zeros(8, 5)
    for call in (lambda: head.rms_norm(x), lambda: head.rms_norm_backward(x, x, x[:, 0]), lambda: head.gated(x, w, w), lambda: head.gated_backward(x[:, :5], x, w, w),
                 lambda: head.adamw([x], [x], head.adamw_moments([x]), 1)):
        with pytest.raises(ValueError):
            call()


def test_moments_at_the_start():
    p = [torch.zeros(3, 50), torch.zeros(0), torch.zeros(129)]
    for (m, v), x in zip(head.adamw_moments(p), p):
        assert m.shape == v.shape == x.shape and m.dtype == v.dtype == torch.float32 and not m.any()
    for (m, ms, v, vs), x, n in zip(head.adamw_moments(p, 8), p, (2, 0, 2)):
        assert m.shape == v.shape == x.shape and m.dtype == v.dtype == head.E4M3 and ms.shape == vs.shape == (n,) and not ms.any() and not m.float().any()
    with pytest.raises(ValueError):
        head.adamw_moments(p, 16)


def test_lists_have_to_match():
    x = torch.zeros(4)
    with pytest.raises(ValueError):
        head.adamw([x], [], [], 1)
    head.adamw([], [], [], 1)
    head.adamw([x], [None], [(x, x)], 1)
