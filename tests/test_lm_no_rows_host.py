"""A gate for every row, of no rows: the calls end before a launch, without a GPU."""
import ctypes

import pytest

A = ctypes.c_void_p(0x1000)      # aligned, never dereferenced
OK, INVALID = 0, 1


@pytest.fixture(scope="module")
def lib():
    from paper_2202_00774_b200 import binding
    return binding.lib()


@pytest.mark.parametrize("rows,groups,status", [(0, 0, OK), (0, 1, OK), (0, 5, OK), (0, -1, INVALID), (4, 0, INVALID)])
def test_no_gates_for_no_rows(lib, rows, groups, status):
    assert lib.sdgp_residual_norm(A, A, A, A, A, rows, 64, groups, 1.0, 1e-6, 0, A, A, None, None, None) == status
    assert lib.sdgp_workspace_size_residual_norm_backward(rows, 64, groups) == 0
    assert lib.sdgp_residual_norm_backward(A, A, A, A, A, A, A, A, A, rows, 64, groups, 1.0, 2, 4, 1, 0, 0, A, A, None, None, None, None, None, A,
                                           1 << 20, None) == status
