"""The language-model layers with weights of another type than the activations: what the pruned contraction reads is the weights rounded to the
type of dL/dO, never their bits."""
import pytest
import torch

from paper_2202_00774_b200.autograd import sdgp_fp8_weights, sdgp_linear_fp8, sdgp_linear_logprob, sdgp_linear_residual_norm

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def random(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).cuda()


@pytest.mark.parametrize("x_type,w_type", [(BF16, FP32), (FP16, FP32), (BF16, FP16), (FP16, BF16)])
@pytest.mark.parametrize("n,m,features", [(2, 4, 192), (1, 8, 256), (3, 4, 128), (4, 4, 64)])
def test_eight_bit_layer(x_type, w_type, n, m, features):
    x, w = random(1, 3, 50, 256).to(x_type).requires_grad_(), (random(2, features, 256) / 16).to(w_type).requires_grad_()
    d = random(3, 3, 50, features).to(x_type)
    y = sdgp_linear_fp8(x, w, n=n, m=m)
    y.backward(d)
    x2, w2 = x.detach().clone().requires_grad_(), w.detach().to(x_type).requires_grad_()
    y2 = sdgp_linear_fp8(x2, w2, sdgp_fp8_weights(w), n=n, m=m)
    y2.backward(d)
    assert torch.equal(y, y2) and torch.equal(x.grad, x2.grad)
    assert w.grad.dtype == w_type and torch.equal(w.grad, w2.grad.to(w_type))


@pytest.mark.parametrize("weight_too", [False, True])
def test_layers_under_autocast(weight_too):
    """fp32 activations and weights, which autocast rounds to bf16 for the forward product."""
    x, w = random(4, 40, 128), random(5, 256, 128) / 11
    t = torch.arange(40, device="cuda")
    residual, pre = random(6, 40, 256).to(BF16), (1 + 0.2 * random(7, 256)).to(BF16)

    def gradients(x, w):
        got = []
        for layer in (lambda a, b: sdgp_linear_logprob(a, b, t), lambda a, b: sdgp_linear_residual_norm(a, b, residual, pre_weight=pre)):
            a, b = x.clone().requires_grad_(), w.clone().requires_grad_(weight_too)
            with torch.autocast("cuda", BF16, enabled=x.dtype == FP32):
                one, two = layer(a, b)
            (one.float().sum() + 0.5 * two.float().square().sum()).backward()
            got += [a.grad] + ([b.grad] if weight_too else [])
        return got

    for a, b in zip(gradients(x, w), gradients(x.to(BF16), w.to(BF16))):
        assert a.dtype == FP32 and torch.equal(a, b.float())
