"""Work memory of the gated pair's gradient where the weights' gradients are not wanted: no partial matrices."""
import ctypes as C

import pytest
import torch

from paper_2309_11071_amd import head
from test_block_arguments import E_ARG, MAX_COLS, MAX_ROWS, gated_grad, lib  # noqa: F401


def test_dx_alone_needs_no_partial_matrices(lib):  # noqa: F811
    for type, size in ((0, 4), (1, 2), (2, 2)):
        ranges = 2 * 36 / 1024 if type == 2 else 0                # float16: 36 bytes for 1024 numbers of 2
        for rows, hidden in ((1, 1), (16, 4096), (64, 64), (65, 3), (300, 100), (33_000, 344), (233_000, 683), (1000, MAX_COLS), (MAX_ROWS, 1), (MAX_ROWS, MAX_COLS)):
            alone = lib.ink_gated_backward_work_dx(rows, hidden, type)
            assert 0 < alone <= 2 ** 30 * (1 + ranges)
            for cols in (1, 128, 602, MAX_COLS):
                all_of_it = lib.ink_gated_backward_work(rows, cols, hidden, type)
                assert alone <= all_of_it
                if rows > 64:
                    assert all_of_it - alone >= 4 * cols * 2 * hidden, "a partial matrix at least"
    assert lib.ink_gated_backward_work_dx(0, 8, 0) == lib.ink_gated_backward_work_dx(4, 0, 0) == lib.ink_gated_backward_work_dx(4, 8, 3) == 0
    assert lib.ink_gated_backward_work_dx(MAX_ROWS + 1, 8, 0) == lib.ink_gated_backward_work_dx(4, MAX_COLS + 1, 0) == 0
    assert tuple(lib.ink_gated_backward_work_dx.argtypes) == (C.c_int64, C.c_int32, C.c_int32)


def test_less_is_refused(lib):  # noqa: F811
    n = lib.ink_gated_backward_work_dx(300, 5, 1)
    assert gated_grad(lib, rows=300, dg=None, du=None, n=n - 1) == E_ARG and "work_dx" in lib.ink_last_error(None).decode()
    for k in (dict(dg=None), dict(du=None), {}):
        assert gated_grad(lib, rows=300, n=n, **k) == E_ARG, "with a weight's gradient the whole of it is needed"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols,hidden", [(3, 40, 50), (300, 70, 33), (9000, 130, 65), (33000, 64, 100)])
def test_nothing_behind_it_is_touched(rows, cols, hidden, dtype):
    g = torch.Generator().manual_seed(rows)
    x, dh = torch.randn(rows, cols, generator=g).to(dtype).cuda(), torch.randn(rows, hidden, generator=g).to(dtype).cuda()
    wg, wu = ((torch.randn(cols, hidden, generator=g) * cols ** -0.5).to(dtype).cuda() for _ in range(2))
    want = head.gated_backward(dh, x, wg, wu)[0]
    assert torch.equal(head.gated_backward(dh, x, wg, wu, need_dweights=False)[0], want)
    lib, t = head._functions(), head.TYPES[dtype]
    n = lib.ink_gated_backward_work_dx(rows, hidden, t)
    work, dx = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda"), torch.empty_like(x)
    assert lib.ink_gated_backward(dh.data_ptr(), hidden, x.data_ptr(), cols, wg.data_ptr(), hidden, wu.data_ptr(), hidden, rows, cols, hidden, t, head.ACTS["silu"], dx.data_ptr(),
                                  cols, None, 0, None, 0, work.data_ptr(), n, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(dx, want) and (work[n:] == 0xA5).all()


@pytest.mark.gpu
def test_a_calls_memory():
    """dx of 100k x 602 x 1605 bfloat16: what the call takes beyond its result, some 650 MB; the partial matrices would be more than 200 MB on top."""
    rows, cols, hidden = 100_000, 602, 1605
    x, dh = torch.randn(rows, cols, device="cuda").bfloat16(), torch.randn(rows, hidden, device="cuda").bfloat16()
    w = (torch.randn(cols, hidden, device="cuda") * cols ** -0.5).bfloat16()
    taken = []
    for weights in (False, True):
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        got = head.gated_backward(dh, x, w, w, need_dweights=weights)
        taken.append(torch.cuda.max_memory_allocated() - before)
        del got
    lib = head._functions()
    step = 2 << 20                                                # torch's allocator takes memory of this size by whole multiples of 2 MiB: dx and the work memory
    assert taken[0] <= lib.ink_gated_backward_work_dx(rows, hidden, 1) + 2 * rows * cols + 2 * step
    assert taken[1] - taken[0] >= lib.ink_gated_backward_work(rows, cols, hidden, 1) - lib.ink_gated_backward_work_dx(rows, hidden, 1) - 2 * step
