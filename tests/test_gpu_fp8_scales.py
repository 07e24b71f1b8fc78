"""The 8-bit product with scales whose product is no normal fp32 number although a block's share of the sum is one: infinite, where the block's
sum is small or zero; subnormal or zero, where it is large. Tolerances as for other scales (tests/test_gpu_fp8.py), with a rounding more for a
block's value, which is then multiplied by the two scales one after the other, and half the smallest number for each block that ends among the
subnormal ones."""
import pytest
import torch

import paper_2202_00774_b200 as sdgp
from paper_2202_00774_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {B.BF16: torch.bfloat16, B.FP32: torch.float32}
E4M3 = torch.float8_e4m3fn
SHAPES = [(1, 128, 512), (5, 130, 400), (20, 256, 1040), (1, 256, 4096), (40, 101, 640), (70, 4099, 384), (300, 520, 640), (600, 1000, 2064)]   # every kernel, split sums too


def spread(s, block_rows, rows, K):
    return s.double().repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :K]


def check(xq, sx, wq, sw, dtype):
    rows, features = xq.shape[0], wq.shape[0]
    y = torch.full((rows, features), 7.0, dtype=TYPES[dtype], device="cuda")
    sdgp.sdgp_fp8_linear(xq, sx, wq, sw, y, dtype=dtype)
    x, w = xq.double() * spread(sx, 1, *xq.shape), wq.double() * spread(sw, 128, *wq.shape)
    want, size = x @ w.t(), x.abs() @ w.abs().t()
    fi = torch.finfo(TYPES[dtype])
    blocks = sx.shape[1]
    tol = (132 + blocks) * 2 ** -23 * size + want.abs() * fi.eps / 2 + fi.smallest_normal * fi.eps + blocks * 2.0 ** -149
    assert torch.isfinite(want).all() and want.abs().max() <= fi.max
    off = (y.double() - want).abs()
    assert torch.all(off <= tol), (off / tol).max()
    assert sdgp.sdgp_last_device_error() == 0
    return want


def numbers(rows, K, seed, tiny=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, K, generator=g) * 60
    if tiny:   # the two smallest numbers, and zero
        x = torch.randint(-2, 3, (rows, K), generator=g) * 2.0 ** -9
    return x.clamp(-448, 448).to(E4M3).cuda()


def scales(rows, blocks, exponent, seed):
    g = torch.Generator().manual_seed(seed)
    return ((1 + torch.rand(rows, blocks, generator=g)) * 2.0 ** exponent).cuda()


@pytest.mark.parametrize("dtype", [B.BF16, B.FP32])
@pytest.mark.parametrize("rows,features,K", SHAPES)
def test_product_of_scales_above_the_range(dtype, rows, features, K):
    blocks, tiles = -(-K // 128), -(-features // 128)
    for ex, ew in ((70, 60), (5, 126), (126, 3)):   # |sums| <= 128 * 2^-16 * K / 128
        want = check(numbers(rows, K, 1, True), scales(rows, blocks, ex, 2), numbers(features, K, 3, True), scales(tiles, blocks, ew, 4), dtype)
        assert want.abs().max() > 2.0 ** 100


@pytest.mark.parametrize("dtype", [B.BF16, B.FP32])
@pytest.mark.parametrize("rows,features,K", SHAPES)
def test_product_of_scales_below_the_range(dtype, rows, features, K):
    blocks, tiles = -(-K // 128), -(-features // 128)
    for ex, ew in ((-80, -56), (-75, -76), (2, -140), (-130, -5)):   # sums of some 2^15
        want = check(numbers(rows, K, 5), scales(rows, blocks, ex, 6), numbers(features, K, 7), scales(tiles, blocks, ew, 8), dtype)
        assert want.abs().max() >= 2.0 ** -138


@pytest.mark.parametrize("dtype", [B.BF16, B.FP32])
@pytest.mark.parametrize("rows,features,K", SHAPES)
def test_blocks_of_zeros_and_ordinary_ones_beside_them(dtype, rows, features, K):
    """Some blocks of some rows: zeros with scales whose product is infinite, large numbers with tiny scales; ordinary ones everywhere else."""
    blocks, tiles = -(-K // 128), -(-features // 128)
    xq, wq = numbers(rows, K, 9), numbers(features, K, 10)
    sx, sw = scales(rows, blocks, -6, 11), scales(tiles, blocks, -6, 12)
    sw[:, 1] = 2.0 ** 100
    xq.view(torch.uint8)[:, 128:256] = 0
    sx[::2, 1] = 1.5 * 2.0 ** 100
    sw[0, 0] = 1.25 * 2.0 ** -100
    sx[::3, 0] = 1.75 * 2.0 ** -40
    sx[rows - 1, blocks - 1] = 0.0
    check(xq, sx, wq, sw, dtype)


@pytest.mark.parametrize("rows,features,K", SHAPES)
def test_other_rows_keep_their_bits(rows, features, K):
    blocks, tiles = -(-K // 128), -(-features // 128)
    xq, wq = numbers(rows, K, 13), numbers(features, K, 14)
    sx, sw = scales(rows, blocks, -6, 15), scales(tiles, blocks, -6, 16)
    y, z = (torch.zeros(rows, features, device="cuda") for _ in range(2))
    sdgp.sdgp_fp8_linear(xq, sx, wq, sw, y, dtype=B.FP32)
    row = rows // 2
    sx[row, blocks // 2] = 2.0 ** -124
    for _ in range(2):
        sdgp.sdgp_fp8_linear(xq, sx, wq, sw, z, dtype=B.FP32)
        others = torch.arange(rows, device="cuda") != row
        assert torch.equal(y[others], z[others])
    x, w = xq.double() * spread(sx, 1, rows, K), wq.double() * spread(sw, 128, features, K)
    tol = (132 + blocks) * 2 ** -23 * (x.abs() @ w.abs().t())[row]
    assert torch.all((z.double()[row] - (x @ w.t())[row]).abs() <= tol)
