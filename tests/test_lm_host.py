"""What the operators around a language model's linear layers refuse, without a GPU: every call below fails (or ends) before a launch."""
import ctypes

import pytest

OK, INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 0, 1, 2, 3, 4
BF16, FP16, FP32 = 0, 1, 2
A = ctypes.c_void_p(0x1000)      # aligned, never dereferenced
ODD = ctypes.c_void_p(0x1002)


@pytest.fixture(scope="module")
def lib():
    from paper_2202_00774_b200 import binding
    return binding.lib()


def logprob(lib, logits=A, targets=A, rows=4, K=64, classes=64, dtype=BF16, top=0, logprob=A, entropy=None, lse=None, top_logprob=None,
            top_token=None):
    return lib.sdgp_token_logprob(logits, targets, rows, K, classes, dtype, top, logprob, entropy, lse, top_logprob, top_token, None)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(dtype=3)), (INVALID, dict(rows=-1)), (INVALID, dict(classes=0)), (INVALID, dict(classes=65)), (INVALID, dict(top=-1)),
    (INVALID, dict(top=65)), (INVALID, dict(logits=None)), (INVALID, dict(targets=None)), (INVALID, dict(logprob=None)),
    (UNSUPPORTED, dict(top=33)), (UNSUPPORTED, dict(K=1 << 31, classes=5)), (UNSUPPORTED, dict(rows=1 << 31)),
    (ALIGNMENT, dict(logits=ODD)), (ALIGNMENT, dict(targets=ctypes.c_void_p(0x1004))), (ALIGNMENT, dict(lse=ODD)),
    (ALIGNMENT, dict(top=3, top_token=ctypes.c_void_p(0x1004))), (OK, dict(rows=0, logits=None, targets=None, logprob=None))])
def test_logprob(lib, status, change):
    assert logprob(lib, **change) == status


def logprob_backward(lib, logits=A, targets=A, lse=A, entropy=None, d_logprob=A, d_entropy=None, rows=4, K=64, classes=64, n=2, m=4, scheme=1,
                     dtype=BF16, grad=A, values=None, meta=None):
    return lib.sdgp_token_logprob_backward(logits, targets, lse, entropy, d_logprob, d_entropy, rows, K, classes, n, m, scheme, 0, dtype,
                                           grad, values, meta, None)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(dtype=7)), (INVALID, dict(rows=-1)), (INVALID, dict(classes=0)), (INVALID, dict(classes=65)), (INVALID, dict(lse=None)),
    (INVALID, dict(d_entropy=A)), (INVALID, dict(values=A, n=0)), (INVALID, dict(values=A, n=5)), (INVALID, dict(values=A, scheme=3)),
    (INVALID, dict(values=A, K=72, m=16)), (UNSUPPORTED, dict(values=A, m=6)), (UNSUPPORTED, dict(values=A, n=3)),
    (UNSUPPORTED, dict(values=A, dtype=FP32)), (ALIGNMENT, dict(values=A, K=72, classes=72, m=8)), (ALIGNMENT, dict(values=ODD)),
    (ALIGNMENT, dict(meta=ODD)), (ALIGNMENT, dict(grad=ODD)), (UNSUPPORTED, dict(rows=(1 << 31) - 1, K=(1 << 31) - 16, classes=5)),
    (OK, dict(grad=None)), (OK, dict(rows=0, logits=None, targets=None, lse=None, grad=None))])
def test_logprob_backward(lib, status, change):
    assert logprob_backward(lib, **change) == status
