"""Rows that are too long for the norm's column arithmetic are refused before anything is launched (host only)."""
import ctypes

import pytest

from paper_2312_00752_b200 import binding as K

a = ctypes.c_void_p(4096)


def _calls(rows, D, io, flags):
    lib = K.load_library()
    p = ctypes.byref(K.ssm_norm_problem_t(rows, D, io, io, flags, 1e-5))
    bias = a if flags & K.SSM_NORM_FLAG_HAS_BIAS else None
    need = lib.ssm_norm_bwd_workspace_bytes(p)
    return (need, lib.ssm_norm_fwd(p, a, None, a, bias, a, None, None, None),
            lib.ssm_norm_bwd(p, a, a, a, a, None, a, None, a, bias, a, 1 << 62, None))


@pytest.mark.parametrize("io", [K.SSM_BF16, K.SSM_F32])
@pytest.mark.parametrize("flags", [0, K.SSM_NORM_FLAG_RMS, K.SSM_NORM_FLAG_HAS_BIAS])
@pytest.mark.parametrize("D", [2 ** 31 - 1, 2 ** 31 - 8, 2 ** 31 - 256, 2 ** 30, 2 ** 28 + 1])
def test_rows_past_the_column_arithmetic_are_refused(D, flags, io):
    assert _calls(1, D, io, flags) == (0, 2, 2)


def test_the_longest_row_and_the_most_rows_are_not():
    lib = K.load_library()
    for rows, D in ((1, 2 ** 28), (2 ** 31 - 1, 1)):
        p = K.ssm_norm_problem_t(rows, D, K.SSM_BF16, K.SSM_BF16, 0, 1e-5)
        assert lib.ssm_norm_bwd_workspace_bytes(ctypes.byref(p)) >= D * 4
    p = K.ssm_norm_problem_t(2 ** 31, 1, K.SSM_BF16, K.SSM_BF16, 0, 1e-5)
    assert lib.ssm_norm_bwd_workspace_bytes(ctypes.byref(p)) == 0
