"""Quantisation to e4m3 with a scale for each block of 128, and the product of two such matrices, against their definitions in 64 bits.

The scale is a power of two, so x / scale is exact and the rounding of the quantisation has one right answer: bits are compared. The product's
terms are exact in fp32; a block's 128 of them are added on the tensor cores, blocks are multiplied by two scales (a rounding each, 2^-24)
and added one after another: (128 + blocks + 3) additions, each off by 2^-23 of the sum of magnitudes at most (the tensor cores' additions
may cut off instead of rounding); y is rounded once, half a step."""
import pytest
import torch

import paper_2202_00774_b200 as sdgp
from paper_2202_00774_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {B.BF16: torch.bfloat16, B.FP16: torch.float16, B.FP32: torch.float32}
E4M3 = torch.float8_e4m3fn


def power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def scales(x, block_rows):
    rows, K = x.shape
    most = torch.nn.functional.pad(x.double().cpu().abs(), (0, -K % 128, 0, -rows % block_rows))
    most = most.unflatten(0, (-1, block_rows)).unflatten(2, (-1, 128)).amax((1, 3))
    e = torch.frexp(most / 448)[1]                       # most / 448 in [2^(e-1), 2^e)
    e = torch.where(most / 448 == power(e - 1), e - 1, e).clamp(min=-126)
    s = torch.where(most == 0, 1.0, power(torch.where(torch.isfinite(most), e, 0)))
    return torch.where(torch.isfinite(most), s, float("nan"))


def spread(s, block_rows, rows, K):
    return s.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :K]


def codes():
    """Every e4m3 number by its code."""
    return torch.arange(256, dtype=torch.uint8).view(E4M3).double()


def rounded(v):
    """Nearest e4m3 numbers, ties to even, from the list of all of them."""
    table = codes()
    pos = table[:127]                                    # 0 .. 448, ascending
    m = v.abs().contiguous()
    hi = torch.searchsorted(pos, m).clamp(1, 126)
    lo = hi - 1
    to_lo, to_hi = m - pos[lo], pos[hi] - m
    pick = torch.where((to_lo < to_hi) | ((to_lo == to_hi) & (lo % 2 == 0)), lo, hi)
    return torch.copysign(pos[pick], v)


def quantize(x, block_rows, dtype):
    q = torch.full(x.shape, 0x55, dtype=torch.uint8, device="cuda").view(E4M3)
    s = torch.full((-(-x.shape[0] // block_rows), -(-x.shape[1] // 128)), 9.0, device="cuda")
    sdgp.sdgp_fp8_quantize(x, q, s, block_rows=block_rows, dtype=dtype)
    return q, s


@pytest.mark.parametrize("dtype", [B.BF16, B.FP16, B.FP32])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,K", [(1, 16), (3, 128), (5, 144), (127, 240), (128, 256), (129, 2112), (300, 1040), (2, 16384), (700, 48)])
def test_quantize(dtype, block_rows, rows, K):
    g = torch.Generator().manual_seed(rows * K)
    x = torch.randn(rows, K, generator=g) * torch.exp2(torch.randint(-12, 6, (rows, 1), generator=g).float())
    if dtype == B.FP32:
        x = x * torch.exp2(torch.randint(-60, 60, (1, K), generator=g).float())
    x = x.to(TYPES[dtype])
    if rows > 2:
        x[1] = 0
        x[2, : min(K, 128)] = 448.0 * 2.0 ** -5     # a largest number that is 448 times a power of two exactly
    x = x.cuda()
    q, s = quantize(x, block_rows, dtype)
    want = scales(x, block_rows)
    assert torch.equal(s.double().cpu(), want)
    v = x.double().cpu() / spread(want, block_rows, rows, K)
    assert torch.equal(q.cpu().double(), rounded(v))


def test_quantize_every_rounding():
    """All e4m3 numbers, the midpoints between neighbours and what lies just beside those."""
    pos = codes()[:127]
    mid = (pos[1:] + pos[:-1]) / 2
    v = torch.cat([pos, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20)])
    v = torch.cat([v, -v])
    x = torch.full((len(v) // 15 + 1, 16), 448.0, dtype=torch.float64)   # 448 in each row: the scale is 1
    flat = x[:, :15].contiguous().view(-1)
    flat[: len(v)] = v
    x[:, :15] = flat.view(-1, 15)
    q, s = quantize(x.float().cuda(), 1, B.FP32)
    assert torch.all(s == 1) and torch.equal(q.cpu().double(), rounded(x.float().double()))


@pytest.mark.parametrize("dtype", [B.BF16, B.FP32])
def test_quantize_numbers_at_the_ends(dtype):
    x = torch.ones(8, 256, dtype=TYPES[dtype])
    x[0, 3], x[1, 130], x[2, 5] = float("nan"), float("inf"), -float("inf")
    x[3] = torch.finfo(TYPES[dtype]).max
    x[4] = torch.finfo(TYPES[dtype]).smallest_normal
    x[5] = torch.finfo(TYPES[dtype]).smallest_normal * torch.finfo(TYPES[dtype]).eps   # the smallest number
    q, s = quantize(x.cuda(), 1, dtype)
    q, s = q.cpu().double(), s.cpu().double()
    want = scales(x, 1)
    assert torch.equal(torch.isnan(s), torch.isnan(want)) and torch.equal(s[3:], want[3:])
    for r, b in ((0, 0), (1, 1), (2, 0)):
        assert torch.isnan(s[r, b]) and torch.isnan(q[r, b * 128:(b + 1) * 128]).all()
        assert s[r, 1 - b] == 2.0 ** -8 and torch.all(q[r, (1 - b) * 128:(2 - b) * 128] == 256)
    assert torch.equal(q[3:], rounded(x[3:].double() / spread(want[3:], 1, 5, 256)))


def operands(rows, features, K, seed):
    g = torch.Generator().manual_seed(seed)
    xq = torch.randn(rows, K, generator=g).mul(60).clamp(-448, 448).to(E4M3)
    wq = torch.randn(features, K, generator=g).mul(60).clamp(-448, 448).to(E4M3)
    sx = torch.rand(rows, -(-K // 128), generator=g) * 0.02 + 1e-3
    sw = torch.rand(-(-features // 128), -(-K // 128), generator=g) * 0.02 + 1e-3
    return xq.cuda(), sx.cuda(), wq.cuda(), sw.cuda()


def product(xq, sx, wq, sw):
    x = xq.double() * spread(sx.double(), 1, *xq.shape)
    w = wq.double() * spread(sw.double(), 128, *wq.shape)
    return x @ w.t(), x.abs() @ w.abs().t()


def check(y, xq, sx, wq, sw, dtype):
    want, size = product(xq, sx, wq, sw)
    fi = torch.finfo(TYPES[dtype])
    tol = (131 + sx.shape[1]) * 2 ** -23 * size + want.abs() * fi.eps / 2 + fi.smallest_normal * fi.eps
    off = (y.double() - want).abs()
    assert torch.all(off <= tol), ((off - tol).max().item(), off.max().item(), torch.nonzero(off > tol)[:5].tolist())


@pytest.mark.parametrize("dtype", [B.BF16, B.FP16, B.FP32])
@pytest.mark.parametrize("rows,features,K", [
    (1, 1, 16), (1, 128, 128), (3, 130, 144), (16, 64, 1024), (17, 256, 2048), (33, 100, 4096), (64, 520, 512), (65, 128, 384), (128, 1000, 272),
    (129, 1001, 1040), (1, 4096, 4096), (40, 2112, 2688), (300, 2048, 640), (777, 1088, 832), (1024, 8192, 512), (2048, 4096, 384),
    (5000, 2064, 144), (4097, 4000, 128), (20, 20000, 4096), (9, 1100, 6000), (33, 64, 16), (300, 24, 5120), (50, 3333, 3344)])
def test_product(dtype, rows, features, K):
    ops = operands(rows, features, K, rows + features + K)
    y = torch.full((rows, features), 7.0, dtype=TYPES[dtype], device="cuda")
    sdgp.sdgp_fp8_linear(*ops, y, dtype=dtype)
    check(y, *ops, dtype)
    again = torch.zeros_like(y)
    sdgp.sdgp_fp8_linear(*ops, again, dtype=dtype)
    assert torch.equal(y, again)
    assert sdgp.sdgp_last_device_error() == 0


def test_product_leaves_what_lies_behind_it():
    for rows, features in ((5, 70), (600, 8200)):
        ops = operands(rows, features, 256, 1)
        whole = torch.full((rows * features + 64,), 3.0, dtype=torch.bfloat16, device="cuda")
        sdgp.sdgp_fp8_linear(*ops, whole[: rows * features].view(rows, features))
        assert torch.all(whole[rows * features:] == 3.0)
        check(whole[: rows * features].view(rows, features), *ops, B.BF16)


def test_product_with_numbers_that_are_not_finite():
    """A NaN scale or element reaches its row (or its features) only."""
    xq, sx, wq, sw = operands(6, 300, 512, 3)
    sx[2, 1] = float("nan")
    wq.view(torch.uint8)[7, 200] = 0x7F
    y = torch.zeros(6, 300, dtype=torch.bfloat16, device="cuda")
    sdgp.sdgp_fp8_linear(xq, sx, wq, sw, y)
    bad = torch.isnan(y)
    assert bad[2].all() and bad[:, 7].all()
    bad[2], bad[:, 7] = False, False
    assert not bad.any()


def test_data_gradient_is_the_product_with_the_transposed_weights():
    """Scales of square blocks are those of the transposed matrix, transposed."""
    g = torch.Generator().manual_seed(4)
    w = torch.randn(384, 256, generator=g).to(torch.bfloat16).cuda()
    d = torch.randn(100, 384, generator=g).to(torch.bfloat16).cuda()
    (wq, sw), (tq, st), (dq, sd) = quantize(w, 128, B.BF16), quantize(w.t().contiguous(), 128, B.BF16), quantize(d, 1, B.BF16)
    assert torch.equal(st, sw.t()) and torch.equal(tq.view(torch.uint8), wq.view(torch.uint8).t())
    y = torch.empty(100, 256, dtype=torch.bfloat16, device="cuda")
    sdgp.sdgp_fp8_linear(dq, sd, tq, st, y)
    check(y, dq, sd, tq, st, B.BF16)
    # each factor's rounding is off by 2^-4 of it at most, or half the smallest step 2^-10 times the scale (below 2^-10 of the block's largest)
    exact = d.double() @ w.double()
    size = d.double().abs() @ w.double().abs()
    assert torch.all((y.double() - exact).abs() <= size * (2 ** -3 + 2 ** -7) + 384 * 2 ** -9 * d.abs().max() * w.abs().max())


def test_streams_and_graphs():
    ops = operands(30, 512, 1024, 9)
    x = torch.randn(30, 1024, device="cuda").to(torch.bfloat16)
    q, s = quantize(x, 1, B.BF16)
    want = torch.zeros(30, 512, dtype=torch.bfloat16, device="cuda")
    sdgp.sdgp_fp8_linear(q, s, ops[2], ops[3], want)
    q2, s2, y = torch.zeros_like(q.view(torch.uint8)), torch.zeros_like(s), torch.zeros_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        sdgp.sdgp_fp8_quantize(x, q2, s2)
        sdgp.sdgp_fp8_linear(q2, s2, ops[2], ops[3], y)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_calls_that_are_refused():
    xq, sx, wq, sw = operands(4, 64, 256, 1)
    y = torch.empty(4, 64, dtype=torch.bfloat16, device="cuda")
    for bad in ((xq[:, :128].contiguous(), sx[:, :1].contiguous(), wq, sw, y), (xq, sx[:3], wq, sw, y), (xq, sx, wq, sw[:, :1].contiguous(), y),
                (xq, sx, wq, sw, y[:, :32].contiguous()), (xq.to(torch.bfloat16), sx, wq, sw, y), (xq, sx.double(), wq, sw, y)):
        with pytest.raises(ValueError):
            sdgp.sdgp_fp8_linear(*bad)
    with pytest.raises(ValueError):
        sdgp.sdgp_fp8_linear(xq, sx, wq, sw, y, dtype=B.FP32)
    with pytest.raises(sdgp.SdgpError):
        sdgp.sdgp_fp8_quantize(torch.zeros(4, 24, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 24, dtype=torch.uint8, device="cuda"), torch.zeros(4, 1, device="cuda"))
    with pytest.raises(sdgp.SdgpError):
        sdgp.sdgp_fp8_quantize(torch.zeros(4, 32, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 32, dtype=torch.uint8, device="cuda"),
                               torch.zeros(1, 1, device="cuda"), block_rows=64)
