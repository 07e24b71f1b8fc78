"""Log probabilities of tokens, entropy and alternatives, and their gradient, against their definitions in 64 bits.

Tolerances. An exponential in the kernels is 2^(d log2 e) with d rounded once and the product once: relative error at most
(1 + |d|) 2^-23 + 2^-22. A row's sums add at most n = V / 256 + 16 terms in sequence in a thread and 13 joins after that, each
addition off by 2^-24 of the sum: (n + 13) 2^-24. Gradients are rounded once to their type: half a step, eps / 2."""
import pytest
import torch

import paper_2202_00774_b200 as sdgp
from paper_2202_00774_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {B.BF16: torch.bfloat16, B.FP16: torch.float16, B.FP32: torch.float32}


def logits_of(rows, K, dtype, seed, scale=2.5):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, K, generator=g) * scale
    t = torch.randint(0, K, (rows,), generator=g)
    return z.to(TYPES[dtype]).cuda(), t.cuda()


def forward(z, t, classes=None, top=0, dtype=B.BF16):
    rows = z.shape[0]
    out = {k: torch.full((rows,), 7.0, device="cuda") for k in ("logprob", "entropy", "lse")}
    if top:
        out["top_logprob"] = torch.full((rows, top), 7.0, device="cuda")
        out["top_token"] = torch.full((rows, top), 7, dtype=torch.int64, device="cuda")
    sdgp.sdgp_token_logprob(z, t, classes=classes, dtype=dtype, **out)
    return {k: v.cpu() for k, v in out.items()}


def definition(z, t, classes=None, top=0):
    z = z[:, :classes].double().cpu()
    t = t.cpu()
    V = z.shape[1]
    most = z.amax(1, keepdim=True)
    empty = (most == -float("inf"))[:, 0]
    w = torch.where(empty[:, None], torch.zeros_like(z), torch.exp(z - most))
    lse = torch.where(empty, -float("inf"), torch.log(w.sum(1)) + most[:, 0])
    p = w / w.sum(1, keepdim=True)
    logp = (z - most) - torch.log(w.sum(1, keepdim=True))   # (with logits of 1e38, lse itself holds nothing of log sum w)
    plogp = torch.where(w == 0, 0.0, p * logp)
    H = torch.where(empty, 0.0, -plogp.sum(1))
    lp = logp.gather(1, t.clamp(0, V - 1)[:, None])[:, 0]
    lp = torch.where(empty, -float("inf"), lp)
    lp = torch.where(t >= V, float("nan"), torch.where(t < 0, 0.0, lp))
    out = {"logprob": lp, "entropy": H, "lse": lse}
    if top:
        order = torch.sort(z, dim=1, descending=True, stable=True)   # equal ones in the order of their index
        out["top_token"] = order.indices[:, :top]
        out["top_logprob"] = torch.where(empty[:, None], -float("inf"), logp.gather(1, order.indices[:, :top]))
    return out


def check(got, want, V, depth=60.0):
    n = V / 256 + 16 + 13
    rel = n * 2 ** -24 + 2 ** -22 + depth * 2 ** -23
    for k in ("logprob", "lse", "top_logprob"):
        if k in want:
            w, g = want[k], got[k].double()
            assert torch.equal(torch.isnan(w), torch.isnan(g)) and torch.equal(torch.isinf(w), torch.isinf(g)), k
            fine = torch.isfinite(w)
            assert torch.all((w - g)[fine].abs() <= rel + 2 ** -22 * w[fine].abs()), (k, (w - g)[fine].abs().max())
    w, g = want["entropy"], got["entropy"].double()
    fine = torch.isfinite(w)
    assert torch.equal(torch.isnan(w), torch.isnan(g))
    assert torch.all((w - g)[fine].abs() <= rel * (2 + 2 * w[fine].abs())), (w - g)[fine].abs().max()
    if "top_token" in want:
        assert torch.equal(got["top_token"], want["top_token"])


@pytest.mark.parametrize("dtype", [B.BF16, B.FP16, B.FP32])
@pytest.mark.parametrize("rows,K,classes,top", [
    (1, 1, 1, 1), (3, 2, 2, 2), (5, 7, 7, 7), (2, 8, 5, 3), (4, 64, 50, 20), (3, 255, 255, 32), (7, 257, 257, 5), (1, 2049, 2049, 32),
    (9, 4099, 4090, 20), (600, 1000, 1000, 4), (2, 50048, 50001, 20), (1, 131072, 131072, 32), (5, 32003, 32003, 1), (300, 2112, 2100, 0), (400, 5000, 4999, 20),
    (1300, 4100, 4100, 7), (1300, 2501, 2501, 0), (200, 9001, 9001, 32), (2, 300000, 299999, 20)])
def test_statistics_and_alternatives(dtype, rows, K, classes, top):
    z, t = logits_of(rows, K, dtype, 17 * rows + K)
    t = t % classes
    if rows > 2:
        t[1] = -100
    check(forward(z, t, classes, top, dtype), definition(z, t, classes, top), classes)


@pytest.mark.parametrize("dtype", [B.BF16, B.FP16, B.FP32])
@pytest.mark.parametrize("K", [40, 1003, 33000])
def test_masks_and_numbers_that_are_not_finite(dtype, K):
    z, t = logits_of(12, K, dtype, K)
    lowest = torch.finfo(TYPES[dtype]).min
    z[0] = -float("inf")                       # nothing left
    z[1, 1:] = -float("inf")                   # one token left
    z[2, ::2] = -float("inf")
    z[3] = lowest                              # the lowest value everywhere: all alike
    z[4, 3:] = lowest
    z[5, K // 2] = float("inf")
    z[6, K - 1] = float("nan")
    z[7, 0] = float("nan")
    z[8] = 0.0
    z[8, 1::2] = -0.0                          # equal to +0: the order is that of the tokens
    t[9], t[10] = -1, K                        # not counted; no token
    t[1], t[2] = 0, 0                          # (the second one has probability 0)
    z[11, : K - 1] = torch.finfo(TYPES[dtype]).max
    top = 20
    got, want = forward(z, t, None, top, dtype), definition(z, t, None, top)
    finite = [0, 1, 2, 3, 8, 9, 10]
    pick = lambda d: {k: v[finite] for k, v in d.items()}
    check(pick(got), pick(want), K)
    for r in (5, 6, 7):
        assert torch.isnan(got["lse"][r]) and torch.isnan(got["entropy"][r]) and torch.isnan(got["logprob"][r])
    assert got["top_token"][5, 0] == K // 2 and not (got["top_token"][6] == K - 1).any() and not (got["top_token"][7] == 0).any()
    for r in (4, 11):
        assert torch.equal(got["top_token"][r, :3], want["top_token"][r, :3])
        assert abs(got["entropy"][r] - want["entropy"][r]) <= (K / 256 + 93) * 2 ** -23 * (2 + 2 * want["entropy"][r])
        assert abs(got["lse"][r].double() - want["lse"][r]) <= (K / 256 + 93) * 2 ** -23 + 2 ** -22 * abs(want["lse"][r])


def test_fewer_numbers_than_alternatives():
    z, t = logits_of(2, 6, B.BF16, 3)
    z[0, 1:5] = float("nan")
    got = forward(z, t, None, 4, B.BF16)
    assert sorted(got["top_token"][0, :2].tolist()) == [0, 5] and got["top_token"][0, 2:].tolist() == [-1, -1]
    assert torch.isnan(got["top_logprob"][0]).all()


@pytest.mark.parametrize("dtype", [B.BF16, B.FP32])
@pytest.mark.parametrize("rows,K,k", [(2, 4096, 32), (1, 70000, 20), (400, 3000, 8), (1300, 5000, 20), (3, 1500, 32), (20, 200000, 32)])
def test_equal_values_go_to_the_lower_token(dtype, rows, K, k):
    """Few distinct values: almost every comparison is a tie; and a row in ascending order, where everything enters the list."""
    g = torch.Generator().manual_seed(K)
    z = torch.randint(-3, 3, (rows, K), generator=g).float()
    z[0] = torch.arange(K) / 7.0
    z = z.to(TYPES[dtype]).cuda()
    t = torch.zeros(rows, dtype=torch.int64, device="cuda")
    got, want = forward(z, t, None, k, dtype), definition(z, t, None, k)
    assert torch.equal(got["top_token"], want["top_token"])


@pytest.mark.parametrize("dtype", [B.BF16, B.FP32])
@pytest.mark.parametrize("rows,K,pad", [(1300, 5000, 0), (1200, 140001, 7), (400, 20000, 3), (150, 300001, 0), (20, 40000, 0), (2, 2500003, 5), (14, 1999, 1)])
def test_alternatives_wherever_the_largest_lie(dtype, rows, K, pad):
    """Rows of every kind: random, one value, descending, ascending, almost all masked, few distinct values, numbers that are none,
    the largest side by side in the middle; parts of a row that one thread reads are one or several rounds."""
    g = torch.Generator(device="cuda").manual_seed(K)
    z = torch.randn(rows, K + pad, generator=g, device="cuda") * 2.5
    ramp = torch.arange(K + pad, device="cuda") / 64.0
    for kind in range(1, 8):
        some = slice(kind if rows > 8 else kind % rows, None, 8)
        if rows <= 8 and kind not in (3, 7):
            continue
        if kind == 1:
            z[some] = 1.5
        elif kind == 2:
            z[some] = -ramp
        elif kind == 3:
            z[some] = ramp
        elif kind == 4:
            z[some, : K // 2] = -float("inf")
            z[some, K // 2 + 11:] = -float("inf")
        elif kind == 5:
            z[some] = torch.round(z[some])
        elif kind == 6:
            z[some, ::3] = float("nan")
        else:
            z[some, K // 2: K // 2 + 77] += 40.0
    z = z.to(TYPES[dtype])
    z[:, K:] = float("inf")                  # behind the classes: not looked at
    t = torch.zeros(rows, dtype=torch.int64, device="cuda")
    numbers = torch.where(torch.isnan(z[:, :K]), -float("inf"), z[:, :K].float())
    order = torch.cat([torch.sort(part, dim=1, descending=True, stable=True).indices[:, :32] for part in numbers.split(64)])
    for top in (1, 20, 32):
        tok = torch.empty(rows, top, dtype=torch.int64, device="cuda")
        lp, out = torch.empty(rows, device="cuda"), torch.empty(rows, top, device="cuda")
        sdgp.sdgp_token_logprob(z, t, lp, classes=K, dtype=dtype, top_token=tok, top_logprob=out)
        assert torch.equal(tok, order[:, :top]), (tok != order[:, :top]).nonzero()[:5]


@pytest.mark.parametrize("rows,K", [(1, 131072), (200, 70000), (500, 30000), (2500, 9000), (3000, 1500)])
def test_alternatives_repeat_themselves(rows, K):
    z, t = logits_of(rows, K, B.BF16, K)
    want = forward(z, t, None, 20, B.BF16)
    for _ in range(20):
        got = forward(z, t, None, 20, B.BF16)
        assert all(torch.equal(got[k], want[k]) for k in want)


def test_outputs_that_are_not_asked_for():
    z, t = logits_of(5, 1000, B.BF16, 1)
    lp = torch.empty(5, device="cuda")
    sdgp.sdgp_token_logprob(z, t, lp)
    assert torch.equal(lp.cpu(), forward(z, t)["logprob"])
    tok = torch.empty(5, 9, dtype=torch.int64, device="cuda")
    sdgp.sdgp_token_logprob(z, t, lp, top_token=tok)
    assert torch.equal(tok.cpu(), forward(z, t, None, 9)["top_token"])


def gradient(z, t, lse, H, g, h, classes):
    z64 = z[:, :classes].double().cpu()
    logp = z64 - lse.double().cpu()[:, None]
    p = torch.exp(logp)
    t = t.cpu()
    g = torch.zeros(len(t), dtype=torch.float64) if g is None else g.double().cpu()
    g = torch.where(t < 0, 0.0, g)
    terms = g[:, None].expand_as(p)
    if h is not None:
        terms = terms + h.double().cpu()[:, None] * (torch.where(p == 0, 0.0, logp) + H.double().cpu()[:, None])
    out = torch.zeros(z.shape, dtype=torch.float64)
    out[:, :classes] = -p * terms
    out[torch.arange(len(t)), t.clamp(min=0)] += torch.where(t < 0, 0.0, g)
    size = p * (g.abs()[:, None] + (h.double().cpu().abs()[:, None] * (logp.abs().clamp(max=1e4) + 1 + H.double().cpu()[:, None].abs()) if h is not None else 0))
    rel = (2 + logp.abs().clamp(max=200)) * 2 ** -22 + 2 ** -21
    slack = torch.zeros_like(out)
    slack[:, :classes] = size * rel
    return out, slack


@pytest.mark.parametrize("dtype", [B.BF16, B.FP16, B.FP32])
@pytest.mark.parametrize("rows,K,classes,g_on,h_on", [
    (1, 1, 1, True, True), (3, 5, 5, True, True), (5, 17, 17, True, False), (4, 64, 50, True, True), (2, 128, 128, False, True),
    (33, 1003, 1003, True, True), (70, 2112, 2100, True, False), (2, 50048, 50001, True, True), (3, 32003, 32003, True, True),
    (2, 64, 64, False, False)])
def test_gradient(dtype, rows, K, classes, g_on, h_on):
    z, t = logits_of(rows, K, dtype, rows + K)
    t = t % classes
    if rows > 2:
        t[2] = -100
    f = forward(z, t, classes, 0, dtype)
    gen = torch.Generator().manual_seed(5)
    g = torch.randn(rows, generator=gen).cuda() if g_on else None
    h = torch.randn(rows, generator=gen).cuda() if h_on else None
    lse, H = f["lse"].cuda(), f["entropy"].cuda()
    grad = torch.full_like(z, 9.0)
    sdgp.sdgp_token_logprob_backward(z, t, lse, g, grad=grad, entropy=H if h_on else None, d_entropy=h, dtype=dtype, classes=classes)
    want, slack = gradient(z, t, lse, H, g, h, classes)
    fi = torch.finfo(TYPES[dtype])
    off = (grad.double().cpu() - want).abs()
    tol = slack * (1 + fi.eps) + want.abs() * fi.eps / 2 + fi.smallest_normal * fi.eps
    tol = tol + 2.0 ** -126 * 1e3    # exponentials below the smallest normal number are zero
    assert torch.all(off <= tol), (off - tol).max()
    assert torch.all(grad[:, classes:] == 0)
    # dL/dO in the place of the logits
    again = z.clone()
    sdgp.sdgp_token_logprob_backward(again, t, lse, g, grad=again, entropy=H if h_on else None, d_entropy=h, dtype=dtype, classes=classes)
    assert torch.equal(again.view(torch.uint8), grad.view(torch.uint8))


def test_gradient_against_differences():
    z, t = logits_of(4, 37, B.FP32, 8, scale=1.0)
    lp, H, lse = (torch.empty(4, device="cuda") for _ in range(3))
    sdgp.sdgp_token_logprob(z, t, lp, entropy=H, lse=lse, dtype=B.FP32)
    g, h = torch.tensor([1.0, -2.0, 0.5, 0.0]).cuda(), torch.tensor([0.0, 1.0, -0.5, 2.0]).cuda()
    grad = torch.empty_like(z)
    sdgp.sdgp_token_logprob_backward(z, t, lse, g, grad=grad, entropy=H, d_entropy=h, dtype=B.FP32)

    def value(x):
        d = definition(x, t)
        return (d["logprob"] * g.cpu().double() + d["entropy"] * h.cpu().double())

    step = 2.0 ** -8
    for j in (0, 5, 36):
        up, down = z.double(), z.double()
        up[:, j] += step
        down[:, j] -= step
        slope = (value(up) - value(down)) / (2 * step)
        # the difference quotient is off by step^2 / 6 times the third derivative, which is below 3 (|g| + 6 |h|) here
        assert torch.all((grad[:, j].double().cpu() - slope).abs() <= step ** 2 / 2 * (g.abs() + 6 * h.abs()).double().cpu() + 1e-6)


def test_gradient_of_rows_without_numbers():
    z, t = logits_of(5, 200, B.BF16, 2)
    z[0] = -float("inf")
    z[1, 7] = float("nan")
    z[2, 0:100] = -float("inf")
    t[2], t[3], t[4] = 5, 200, -7
    f = forward(z, t)
    g = torch.ones(5, device="cuda")
    grad = torch.empty_like(z)
    sdgp.sdgp_token_logprob_backward(z, t, f["lse"].cuda(), g, grad=grad, entropy=f["entropy"].cuda(), d_entropy=g, dtype=B.BF16)
    assert torch.all(grad[0] == 0) and torch.isnan(grad[1]).all() and torch.isnan(grad[3]).all()
    assert torch.isfinite(grad[2]).all() and torch.all(grad[2, :5] == 0) and grad[2, 5] == 1 and torch.isfinite(grad[4]).all()


@pytest.mark.parametrize("dtype", [B.BF16, B.FP16])
@pytest.mark.parametrize("n,m", [(1, 4), (2, 4), (1, 8), (2, 8), (1, 16), (2, 16), (1, 32), (2, 32)])
@pytest.mark.parametrize("scheme", [B.RANDOM, B.MAGNITUDE, B.RESCALED_MAGNITUDE])
def test_pruned_copy_is_algorithm_1_on_the_gradient(dtype, n, m, scheme):
    for rows, K, classes in ((3, 160, 150), (37, 2112, 2112), (3, 8224, 8200), (2, 20000, 20000)):
        z, t = logits_of(rows, K, dtype, n * m)
        f = forward(z, t % classes, classes, 0, dtype)
        g = torch.randn(rows, device="cuda")
        args = dict(entropy=f["entropy"].cuda(), d_entropy=g, n=n, m=m, scheme=scheme, seed=99, dtype=dtype, classes=classes)
        grad = torch.empty_like(z)
        out = [(torch.zeros(rows, K // 2, dtype=z.dtype, device="cuda"), torch.zeros(rows, K // 16, dtype=torch.int16, device="cuda")) for _ in range(3)]
        sdgp.sdgp_token_logprob_backward(z, t % classes, f["lse"].cuda(), g, grad=grad, values=out[0][0], meta=out[0][1], **args)
        sdgp.sdgp_token_logprob_backward(z, t % classes, f["lse"].cuda(), g, values=out[1][0], meta=out[1][1], **args)
        sdgp.sdgp_prune_typed(grad, n, m, scheme, 99, dtype, values=out[2][0], meta=out[2][1])
        for v, e in out[:2]:
            assert torch.equal(v.view(torch.int16), out[2][0].view(torch.int16)) and torch.equal(e, out[2][1])


def test_streams_and_graphs():
    z, t = logits_of(40, 5000, B.BF16, 4)
    want = forward(z, t, None, 5)
    side = torch.cuda.Stream()
    out = [torch.zeros(40, device="cuda") for _ in range(3)]
    tok, val = torch.zeros(40, 5, dtype=torch.int64, device="cuda"), torch.zeros(40, 5, device="cuda")
    grad = torch.zeros_like(z)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    g = torch.ones(40, device="cuda")
    with torch.cuda.graph(graph, stream=side):
        sdgp.sdgp_token_logprob(z, t, out[0], entropy=out[1], lse=out[2], top_logprob=val, top_token=tok)
        sdgp.sdgp_token_logprob_backward(z, t, out[2], g, grad=grad, entropy=out[1], d_entropy=g)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0].cpu(), want["logprob"]) and torch.equal(tok.cpu(), want["top_token"]) and torch.equal(val.cpu(), want["top_logprob"])
    ref = torch.zeros_like(z)
    sdgp.sdgp_token_logprob_backward(z, t, out[2], g, grad=ref, entropy=out[1], d_entropy=g)
    assert torch.equal(ref, grad)


def test_two_streams_at_once():
    both = [logits_of(300, 20000, B.BF16, k) for k in (21, 22)]
    want = [forward(z, t, None, 10) for z, t in both]
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    torch.cuda.synchronize()
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                out = [torch.empty(300, device="cuda") for _ in range(3)]
                tok = torch.empty(300, 10, dtype=torch.int64, device="cuda")
                sdgp.sdgp_token_logprob(*both[k], out[0], entropy=out[1], lse=out[2], top_token=tok)
                got[k].append((out, tok))
    torch.cuda.synchronize()
    for k in range(2):
        for out, tok in got[k]:
            assert torch.equal(out[0].cpu(), want[k]["logprob"]) and torch.equal(out[1].cpu(), want[k]["entropy"]) and torch.equal(tok.cpu(), want[k]["top_token"])


def test_calls_that_are_refused():
    z, t = logits_of(4, 64, B.BF16, 1)
    lp = torch.empty(4, device="cuda")
    for bad in (dict(dtype=B.FP32), dict(classes=0), dict(classes=65), dict(top_token=torch.empty(4, 40, dtype=torch.int64, device="cuda")),
                dict(lse=torch.empty(3, device="cuda")), dict(entropy=torch.empty(4, dtype=torch.float64, device="cuda")),
                dict(top_token=torch.empty(4, 4, dtype=torch.int64, device="cuda"), top_logprob=torch.empty(4, 3, device="cuda"))):
        with pytest.raises((ValueError, sdgp.SdgpError)):
            sdgp.sdgp_token_logprob(z, t, lp, **bad)
    with pytest.raises(ValueError):
        sdgp.sdgp_token_logprob(z.t(), t, lp)
    with pytest.raises(ValueError):
        sdgp.sdgp_token_logprob(z, t.int(), lp)
    with pytest.raises(sdgp.SdgpError):    # an entropy gradient without the entropy
        sdgp.sdgp_token_logprob_backward(z, t, lp, lp, grad=z.clone(), d_entropy=lp)
    z32 = z.float()
    with pytest.raises(sdgp.SdgpError):    # fp32 gradients have no compressed form
        sdgp.sdgp_token_logprob_backward(z32, t, lp, lp, values=torch.empty(4, 32, dtype=torch.bfloat16, device="cuda"), dtype=B.FP32)
