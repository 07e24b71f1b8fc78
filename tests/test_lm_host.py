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


def norm(lib, branch=A, residual=A, post_weight=A, gate=A, pre_weight=A, rows=4, C=64, groups=1, dtype=BF16, out=A, y=A, post_rstd=None,
         pre_rstd=None):
    return lib.sdgp_residual_norm(branch, residual, post_weight, gate, pre_weight, rows, C, groups, 1.0, 1e-6, dtype, out, y, post_rstd,
                                  pre_rstd, None)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(dtype=3)), (INVALID, dict(rows=-1)), (INVALID, dict(C=0)), (INVALID, dict(groups=0)), (INVALID, dict(groups=3)),
    (INVALID, dict(branch=None)), (INVALID, dict(residual=None)), (INVALID, dict(out=None)), (INVALID, dict(y=None)),
    (INVALID, dict(pre_weight=None)), (UNSUPPORTED, dict(C=(1 << 24) + 1)), (UNSUPPORTED, dict(rows=(1 << 28) + 1)),
    (ALIGNMENT, dict(branch=ODD)), (ALIGNMENT, dict(gate=ODD)), (ALIGNMENT, dict(y=ODD)), (ALIGNMENT, dict(pre_rstd=ODD)),
    (OK, dict(rows=0, branch=None, residual=None, out=None, y=None))])
def test_norm(lib, status, change):
    assert norm(lib, **change) == status


def norm_backward(lib, branch=A, out=A, d_out=A, d_y=A, post_weight=A, gate=A, pre_weight=A, post_rstd=A, pre_rstd=A, rows=4, C=64, groups=1,
                  n=2, m=4, scheme=1, dtype=BF16, d_residual=A, d_branch=A, d_gate=A, d_post_weight=A, d_pre_weight=A, values=None, meta=None,
                  workspace=A, size=None):
    if size is None:
        size = lib.sdgp_workspace_size_residual_norm_backward(rows, C, groups) if rows > 0 and C > 0 and groups > 0 else 1 << 20
    return lib.sdgp_residual_norm_backward(branch, out, d_out, d_y, post_weight, gate, pre_weight, post_rstd, pre_rstd, rows, C, groups, 1.0,
                                           n, m, scheme, 0, dtype, d_residual, d_branch, d_gate, d_post_weight, d_pre_weight, values, meta,
                                           workspace, size, None)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(dtype=3)), (INVALID, dict(rows=-1)), (INVALID, dict(C=0)), (INVALID, dict(groups=3)), (INVALID, dict(branch=None)),
    (INVALID, dict(d_out=None, d_y=None, d_pre_weight=None)), (INVALID, dict(out=None)), (INVALID, dict(pre_weight=None, d_pre_weight=None)),
    (INVALID, dict(pre_rstd=None)), (INVALID, dict(post_rstd=None)), (INVALID, dict(gate=None)), (INVALID, dict(post_weight=None)),
    (INVALID, dict(d_y=None)), (INVALID, dict(values=A, n=5)), (UNSUPPORTED, dict(values=A, n=3)), (UNSUPPORTED, dict(meta=A, dtype=FP32)),
    (ALIGNMENT, dict(values=A, C=40, m=8)), (ALIGNMENT, dict(d_residual=ODD)), (ALIGNMENT, dict(d_gate=ODD)),
    (WORKSPACE, dict(workspace=None)), (WORKSPACE, dict(workspace=ctypes.c_void_p(0x1010))), (WORKSPACE, dict(size=16))])
def test_norm_backward(lib, status, change):
    assert norm_backward(lib, **change) == status


def test_norm_backward_workspace(lib):
    size = lib.sdgp_workspace_size_residual_norm_backward
    assert size(0, 64, 1) == 0 and size(4, 0, 1) == 0 and size(4, 64, 3) == 0
    assert size(1, 64, 1) >= 2 * 64 * 4 and size(1 << 20, 4096, 1) < 1 << 24
    assert size(30000, 1001, 10000) <= 30000 * 1001 * 4 + (1 << 24)   # sums of a gate for three rows each


def quantize(lib, x=A, rows=4, K=64, block_rows=1, dtype=BF16, q=A, scale=A):
    return lib.sdgp_fp8_quantize(x, rows, K, block_rows, dtype, q, scale, None)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(dtype=3)), (INVALID, dict(rows=-1)), (INVALID, dict(K=-16)), (INVALID, dict(x=None)), (INVALID, dict(q=None)),
    (INVALID, dict(scale=None)), (UNSUPPORTED, dict(block_rows=64)), (UNSUPPORTED, dict(rows=1 << 31)), (ALIGNMENT, dict(K=40)),
    (ALIGNMENT, dict(x=ODD)), (ALIGNMENT, dict(q=ODD)), (ALIGNMENT, dict(scale=ODD)), (OK, dict(rows=0, x=None)), (OK, dict(K=0, x=None)),
    (UNSUPPORTED, dict(rows=(1 << 31) - 1, K=(1 << 31) - 16))])
def test_quantize(lib, status, change):
    assert quantize(lib, **change) == status


def linear(lib, xq=A, x_scale=A, wq=A, w_scale=A, y=A, rows=4, features=64, K=64, dtype=BF16):
    return lib.sdgp_fp8_linear(xq, x_scale, wq, w_scale, y, rows, features, K, dtype, None)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(dtype=3)), (INVALID, dict(rows=-1)), (INVALID, dict(features=-1)), (INVALID, dict(K=0)), (INVALID, dict(xq=None)),
    (INVALID, dict(x_scale=None)), (INVALID, dict(wq=None)), (INVALID, dict(w_scale=None)), (INVALID, dict(y=None)),
    (UNSUPPORTED, dict(rows=1 << 31)), (ALIGNMENT, dict(K=40)), (ALIGNMENT, dict(xq=ODD)), (ALIGNMENT, dict(y=ODD)),
    (ALIGNMENT, dict(w_scale=ODD)), (OK, dict(rows=0, xq=None)), (OK, dict(features=0, wq=None))])
def test_fp8_linear(lib, status, change):
    assert linear(lib, **change) == status


def test_quantized_weights_of_another_shape_are_refused():
    import torch
    from paper_2202_00774_b200.autograd import sdgp_linear_fp8
    x, w = torch.zeros(2, 128, dtype=torch.bfloat16), torch.zeros(256, 128, dtype=torch.bfloat16)
    q, scale = torch.zeros(128, 128, dtype=torch.uint8), torch.ones(1, 1)
    with pytest.raises(ValueError, match="shape"):
        sdgp_linear_fp8(x, w, quantized=(q, scale))
