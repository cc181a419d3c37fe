"""The ends of the ranges that an answer head's operators take, at the C boundary: no launch happens, so no GPU is needed."""
import os

import pytest

from paper_2309_11071_amd import binding

M = 1 << 20          # an address that nothing reads
MAX_CLASSES, MAX_TOP, MAX_COLS, MAX_ROWS = 1 << 27, 16, 16384, (1 << 31) - 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.lib_path()):
        pytest.skip("libink.so not built")
    from paper_2309_11071_amd import head
    return head._functions()


def probs(lib, classes, rows=4, top=0, work=0):
    return lib.ink_log_probs(M, classes, None, 0, rows, classes, 1, 1.0, top, M, M, M, M, M, M, work, None)


def test_the_most_classes(lib):
    assert lib.ink_log_probs_work(4, MAX_CLASSES, 1, MAX_TOP) > 0
    assert lib.ink_log_probs_work(4, MAX_CLASSES + 1, 1, MAX_TOP) == 0 and lib.ink_log_probs_work(4, MAX_CLASSES, 1, MAX_TOP + 1) == 0
    assert probs(lib, MAX_CLASSES) == 1 and "work" in lib.ink_last_error(None).decode(), "the classes are in range, the work memory is not there"
    assert probs(lib, MAX_CLASSES, rows=0) == 0
    for rows in (0, 4):
        assert probs(lib, MAX_CLASSES + 1, rows=rows) == 1 and "classes" in lib.ink_last_error(None).decode()
    assert probs(lib, 100_000, top=MAX_TOP) == 1 and "work" in lib.ink_last_error(None).decode()
    assert probs(lib, 100_000, top=MAX_TOP + 1) == 1 and "top" in lib.ink_last_error(None).decode()
    back = lambda classes: lib.ink_log_probs_backward(None, 1, None, 0, None, None, None, None, 0, classes, 1, 1.0, None, 1, None)   # noqa: E731
    assert back(MAX_CLASSES) == 0 and back(MAX_CLASSES + 1) == 1


def test_the_widest_rows(lib):
    norm = lambda cols, rows=0: lib.ink_layer_norm(None, cols, None, None, rows, cols, 0, 0, 1e-5, None, cols, None, None, None)   # noqa: E731
    linear = lambda cols, out: lib.ink_linear(None, cols, M, out, None, None, 0, 0, cols, out, 1, 1, 0, None, out, None, 0, None)  # noqa: E731
    assert norm(MAX_COLS) == 0 and norm(MAX_COLS + 1) == 1 and norm(8, MAX_ROWS + 1) == 1
    assert linear(MAX_COLS, MAX_COLS) == 0 and linear(MAX_COLS + 1, 8) == 1 and linear(8, MAX_COLS + 1) == 1
    assert lib.ink_linear_backward_work(1, MAX_COLS, MAX_COLS) > 0 and lib.ink_linear_backward_work(1, MAX_COLS + 1, 8) == 0
    assert lib.ink_layer_norm_backward_work(MAX_ROWS, MAX_COLS, 0) > 0 and lib.ink_layer_norm_backward_work(MAX_ROWS + 1, 8, 0) == 0


def test_the_largest_scale(lib):
    """The scale's product with log2 e has to be a number."""
    def call(scale):
        return (lib.ink_log_probs(None, 8, None, 0, 0, 8, 0, scale, 0, None, None, None, None, None, None, 0, None),
                lib.ink_log_probs_backward(None, 8, None, 0, None, None, None, None, 0, 8, 0, scale, None, 8, None))
    assert call(2.3e38) == (0, 0)
    assert call(2.4e38) == (1, 1) and "scale" in lib.ink_last_error(None).decode()
