"""Element types that are not the ones that `dtype` names are refused: their bits would be read as other numbers. Integers of 16 bits (and, for
e4m3 numbers, unsigned bytes) are taken as the numbers' bits, as everywhere in this library."""
import pytest
import torch

import paper_2202_00774_b200 as sdgp
from paper_2202_00774_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {B.BF16: torch.bfloat16, B.FP16: torch.float16, B.FP32: torch.float32}
OTHERS = [(B.BF16, torch.float16), (B.FP16, torch.bfloat16), (B.FP32, torch.int32), (B.BF16, torch.float32), (B.FP32, torch.float16)]


def f32(*shape):
    return torch.zeros(*shape, device="cuda")


@pytest.mark.parametrize("dtype,other", OTHERS)
def test_log_probabilities(dtype, other):
    z, t = f32(4, 64).to(TYPES[dtype]), torch.zeros(4, dtype=torch.int64, device="cuda")
    wrong = f32(4, 64).to(other)
    with pytest.raises(ValueError):
        sdgp.sdgp_token_logprob(wrong, t, f32(4), dtype=dtype)
    with pytest.raises(ValueError):
        sdgp.sdgp_token_logprob_backward(wrong, t, f32(4), f32(4), grad=z.clone(), dtype=dtype)
    with pytest.raises(ValueError):
        sdgp.sdgp_token_logprob_backward(z, t, f32(4), f32(4), grad=wrong, dtype=dtype)
    if dtype != B.FP32:
        with pytest.raises(ValueError):
            sdgp.sdgp_token_logprob_backward(z, t, f32(4), f32(4), values=f32(4, 32).to(other), dtype=dtype)


@pytest.mark.parametrize("dtype,other", OTHERS)
def test_block_boundary(dtype, other):
    type_ = TYPES[dtype]
    good = dict(branch=f32(4, 64).to(type_), residual=f32(4, 64).to(type_), out=f32(4, 64).to(type_), y=f32(4, 64).to(type_),
                post_weight=f32(64).to(type_), gate=f32(1, 64).to(type_), pre_weight=f32(64).to(type_))
    sdgp.sdgp_residual_norm(**good, dtype=dtype)
    for name, t in good.items():
        with pytest.raises(ValueError):
            sdgp.sdgp_residual_norm(**{**good, name: t.to(other)}, dtype=dtype)
    ws = torch.empty(sdgp.sdgp_workspace_size_residual_norm_backward(4, 64, 1), dtype=torch.uint8, device="cuda")
    good = dict(branch=good["branch"], out=good["out"], d_out=f32(4, 64).to(type_), d_y=f32(4, 64).to(type_), post_weight=good["post_weight"],
                gate=good["gate"], pre_weight=good["pre_weight"], d_residual=f32(4, 64).to(type_), d_branch=f32(4, 64).to(type_))
    rest = dict(post_rstd=f32(4), pre_rstd=f32(4), dtype=dtype, workspace=ws)
    sdgp.sdgp_residual_norm_backward(**good, **rest)
    for name, t in good.items():
        with pytest.raises(ValueError):
            sdgp.sdgp_residual_norm_backward(**{**good, name: t.to(other)}, **rest)


@pytest.mark.parametrize("other", [torch.float8_e5m2, torch.int8, torch.bool])
def test_eight_bit_numbers(other):
    q, scale = torch.zeros(4, 128, dtype=torch.uint8, device="cuda"), f32(4, 1)
    wrong = torch.zeros(4, 128, device="cuda").to(other)
    x, y = f32(4, 128).bfloat16(), f32(4, 4).bfloat16()
    with pytest.raises(ValueError):
        sdgp.sdgp_fp8_quantize(x, wrong, scale)
    for pair in ((wrong, q), (q, wrong)):
        with pytest.raises(ValueError):
            sdgp.sdgp_fp8_linear(pair[0], scale, pair[1], f32(1, 1), y)
    for dtype, type_ in ((B.BF16, torch.float16), (B.FP16, torch.bfloat16)):
        with pytest.raises(ValueError):
            sdgp.sdgp_fp8_quantize(x.to(type_), q, scale, dtype=dtype)
        with pytest.raises(ValueError):
            sdgp.sdgp_fp8_linear(q, scale, q, f32(1, 1), y.to(type_), dtype=dtype)


@pytest.mark.parametrize("dtype", [B.BF16, B.FP16])
def test_bits_are_taken(dtype):
    z = torch.randn(4, 200, generator=torch.Generator().manual_seed(1)).to(TYPES[dtype]).cuda()
    t = torch.arange(4, device="cuda")
    want, got = f32(4), f32(4)
    sdgp.sdgp_token_logprob(z, t, want, dtype=dtype)
    for bits in (torch.int16, torch.uint16):
        got.zero_()
        sdgp.sdgp_token_logprob(z.view(bits), t, got, dtype=dtype)
        assert torch.equal(got, want)
    x = torch.randn(3, 128, generator=torch.Generator().manual_seed(2)).to(TYPES[dtype]).cuda()
    q = [torch.zeros(3, 128, dtype=d, device="cuda") for d in (torch.float8_e4m3fn, torch.uint8)]
    for out in q:
        sdgp.sdgp_fp8_quantize(x, out, f32(3, 1), dtype=dtype)
    assert torch.equal(q[0].view(torch.uint8), q[1])
