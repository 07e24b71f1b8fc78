"""The language-model layers on a batch without rows."""
import pytest
import torch

from paper_2202_00774_b200.autograd import sdgp_linear_fp8, sdgp_linear_logprob, sdgp_linear_residual_norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(0,), (0, 7), (2, 0)])
@pytest.mark.parametrize("gates", ["none", "one", "each"])
def test_layers_of_no_rows(shape, gates):
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda").requires_grad_()
    x, residual, w = z(*shape, 128), z(*shape, 256), z(256, 128)
    post, pre, gate = z(256), z(256), {"none": None, "one": z(1, 256), "each": z(*shape, 256)}[gates]
    up = sdgp_linear_fp8(x, w)
    out, y = sdgp_linear_residual_norm(x, w, residual, post, pre, gate)
    lp, entropy = sdgp_linear_logprob(x, w, torch.zeros(*shape, dtype=torch.int64, device="cuda"))
    assert up.shape == out.shape == y.shape == (*shape, 256) and lp.shape == entropy.shape == shape
    (up.sum() + out.sum() + y.sum() + lp.sum() + entropy.sum()).backward()
    for t in (x, residual, w, post, pre) + ((gate,) if gate is not None else ()):
        assert t.grad.shape == t.shape and torch.all(t.grad == 0)
