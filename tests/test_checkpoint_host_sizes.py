"""Sizes whose buffers no 64-bit count holds are refused before a device is looked at; nothing here needs a GPU."""
import ctypes as C

import pytest

MOST_ROWS, MOST_COLS = 2 ** 31 - 1, 2 ** 30 - 1
A = 1 << 20   # an aligned address that nothing reads


@pytest.mark.parametrize("dtype,samples,rows,cols,outs", [(0, 1, MOST_ROWS, 32, MOST_COLS), (1, 1, MOST_ROWS, 2 ** 24, 32), (0, MOST_ROWS, 0, 2 ** 24, 2 ** 20),
                                                          (1, MOST_ROWS, 1, 2 ** 22, 2 ** 20)])
def test_weight_gradients_beyond_all_memory(ampq, dtype, samples, rows, cols, outs):
    """Workspaces and gradients of more than 2^52 bytes: the workspace query's sum of them had wrapped to a negative number,
    and the call then asked for no workspace at all."""
    L, n = ampq.lib(), C.c_longlong()
    groups = -(-cols // 32)
    assert L.ampq_ckpt_weight_grad_workspace(0, dtype, A, outs, samples, rows, cols, outs, C.byref(n)) == ampq.ERR_TOO_LARGE
    assert L.ampq_ckpt_weight_grad(0, None, dtype, 1, A, outs, A, groups * 32, A, groups, samples, rows, cols, outs, A, 0, 0, 0) == ampq.ERR_TOO_LARGE


def test_the_largest_of_each_size_is_allowed(ampq):
    L, n = ampq.lib(), C.c_longlong()
    for dtype, samples, rows, cols, outs in ((0, 1, MOST_ROWS, 64, 64), (1, MOST_ROWS, 1, 64, 64), (0, 1, 300, MOST_COLS, 64), (1, 1, 300, 64, MOST_COLS)):
        assert L.ampq_ckpt_weight_grad_workspace(0, dtype, A, outs, samples, rows, cols, outs, C.byref(n)) in (ampq.OK, ampq.ERR_CUDA)
