"""The layers of a language model together: 8-bit and pruned linear layers, block boundaries, the head; forward and backward as a training
step uses them."""
import pytest
import torch

import paper_2202_00774_b200 as sdgp
from paper_2202_00774_b200 import binding as B
from paper_2202_00774_b200.autograd import (sdgp_fp8_weights, sdgp_linear, sdgp_linear_fp8, sdgp_linear_logprob, sdgp_linear_residual_norm)

pytestmark = pytest.mark.gpu

ALPHA, EPS = 0.75, 1e-6


def parameters(C, H, V, blocks, groups, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    p = []
    for _ in range(blocks):
        p.append({"up": r(H, C) / C ** 0.5, "down": r(C, H) / H ** 0.5, "post": 1 + 0.2 * r(C), "pre": 1 + 0.2 * r(C), "gate": 0.5 + 0.2 * r(groups, C)})
    head = r(V, C) / C ** 0.5 * 2
    p = [{k: v.to(dtype).cuda().requires_grad_() for k, v in b.items()} for b in p]
    return p, head.to(dtype).cuda().requires_grad_()


def network(x, targets, blocks, head, classes, n, m, fp8=False, seed=0):
    stream, y = x, x
    for b in blocks:
        up = sdgp_linear_fp8(y, b["up"], n=n, m=m, seed=seed) if fp8 else sdgp_linear(y, b["up"], n, m, seed=seed)
        stream, y = sdgp_linear_residual_norm(torch.relu(up), b["down"], stream, b["post"], b["pre"], b["gate"], ALPHA, EPS, n=n, m=m, seed=seed)
    return sdgp_linear_logprob(y, head, targets, classes, n=n, m=m, seed=seed)


def plain(x, targets, blocks, head, classes):
    """The same network in 64 bits, out of elementary operations that autograd differentiates."""
    norm = lambda v, w: v * (v.square().mean(-1, keepdim=True) + EPS) ** -0.5 * w
    stream = y = x
    rows = x.shape[0]
    for b in blocks:
        branch = torch.relu(y @ b["up"].t()) @ b["down"].t()
        gate = b["gate"].repeat_interleave(rows // b["gate"].shape[0], 0)
        stream = ALPHA * stream + gate * norm(branch, b["post"])
        y = norm(stream, b["pre"])
    z = (y @ head.t())[:, :classes]
    logp = torch.log_softmax(z, 1)
    lp = torch.where(targets < 0, 0.0, logp.gather(1, targets.clamp(min=0)[:, None])[:, 0])
    return lp, -(logp.exp() * logp).sum(1)


@pytest.mark.parametrize("groups", [1, 4, 96])
def test_without_pruning_the_gradients_are_the_networks(groups):
    """n == m prunes nothing. Rounding each of the two blocks' and the head's tensors to binary16 (2^-11 of a value each) happens some 10
    times on the way of a gradient forward and 10 times back; a gradient's norm is off by 20 of them, times the network's amplification of
    a disturbance, taken as 4."""
    rows, C, H, V, classes = 96, 128, 256, 384, 370
    blocks, head = parameters(C, H, V, 2, groups, torch.float16, 1)
    g = torch.Generator().manual_seed(2)
    x = torch.randn(rows, C, generator=g).half().cuda().requires_grad_()
    t = torch.randint(0, classes, (rows,), generator=g).cuda()
    t[5] = -100
    weights = torch.rand(rows, generator=g).cuda()
    lp, H_ = network(x, t, blocks, head, classes, 4, 4)
    scale = 256.0   # (gradients of binary16 without loss scaling underflow)
    (scale * (weights * (-lp - 0.1 * H_)).mean()).backward()
    leaves = [x, head] + [v for b in blocks for v in b.values()]
    twins = [v.detach().double().requires_grad_() for v in leaves]
    names = list(blocks[0])
    tb = [dict(zip(names, twins[2 + 5 * i: 7 + 5 * i])) for i in range(2)]
    lp2, H2 = plain(twins[0], t, tb, twins[1], classes)
    (scale * (weights.double() * (-lp2 - 0.1 * H2)).mean()).backward()
    assert (lp.double() - lp2).norm() <= 4 * 10 * 2 ** -11 * lp2.norm()
    assert (H_.double() - H2).norm() <= 4 * 10 * 2 ** -11 * H2.norm()
    for a, b in zip(leaves, twins):
        assert a.grad.dtype == a.dtype and a.grad.shape == a.shape
        assert (a.grad.double() - b.grad).norm() <= 4 * 20 * 2 ** -11 * b.grad.norm(), (a.shape, (a.grad.double() - b.grad).norm() / b.grad.norm())


def test_pruned_gradients_are_the_calls_one_after_another():
    """The layers' pruned backward pass, bit for bit, from the library's calls made by hand."""
    rows, C, H, V, n, m, seed = 80, 256, 128, 512, 2, 4, 7
    blocks, head = parameters(C, H, V, 1, 2, torch.bfloat16, 3)
    b = blocks[0]
    gen = torch.Generator().manual_seed(4)
    x = torch.randn(rows, C, generator=gen).bfloat16().cuda().requires_grad_()
    h = torch.relu(torch.randn(rows, H, generator=gen)).bfloat16().cuda().requires_grad_()
    t = torch.randint(0, V, (rows,), generator=gen).cuda()
    out, y = sdgp_linear_residual_norm(h, b["down"], x, b["post"], b["pre"], b["gate"], ALPHA, EPS, n=n, m=m, seed=seed)
    lp, H_ = sdgp_linear_logprob(y, head, t, n=n, m=m, seed=seed)
    (-(lp.sum()) - 0.5 * H_.sum() + out.float().sum()).backward()

    f = lambda *s: torch.empty(*s, device="cuda")
    logits = y.detach() @ head.detach().t()
    lse, ent, lp2 = f(rows), f(rows), f(rows)
    sdgp.sdgp_token_logprob(logits, t, lp2, entropy=ent, lse=lse)
    assert torch.equal(lp2, lp)
    dz, vals, meta = torch.empty_like(logits), f(rows, V // 2).bfloat16(), torch.empty(rows, V // 16, dtype=torch.int16, device="cuda")
    sdgp.sdgp_token_logprob_backward(logits, t, lse, torch.full((rows,), -1.0, device="cuda"), grad=dz, entropy=ent,
                                     d_entropy=torch.full((rows,), -0.5, device="cuda"), n=n, m=m, seed=seed, values=vals, meta=meta)
    dy = torch.empty(rows, C, dtype=torch.bfloat16, device="cuda")
    sdgp.sdgp_spmm_linear(vals, meta, head.detach(), dy)
    assert torch.equal(head.grad, dz.t() @ y.detach())
    branch = h.detach() @ b["down"].detach().t()
    pr, qr, o2, y2 = f(rows), f(rows), torch.empty_like(branch), torch.empty_like(branch)
    w = {k: v.detach() for k, v in b.items()}
    sdgp.sdgp_residual_norm(branch, x.detach(), o2, y2, post_weight=w["post"], gate=w["gate"], pre_weight=w["pre"], alpha=ALPHA, eps=EPS, post_rstd=pr, pre_rstd=qr)
    assert torch.equal(o2, out) and torch.equal(y2, y)
    got = {"d_residual": torch.empty_like(branch), "d_branch": torch.empty_like(branch), "d_gate": f(2, C), "d_post_weight": f(C), "d_pre_weight": f(C)}
    vals, meta = f(rows, C // 2).bfloat16(), torch.empty(rows, C // 16, dtype=torch.int16, device="cuda")
    ws = torch.empty(sdgp.sdgp_workspace_size_residual_norm_backward(rows, C, 2), dtype=torch.uint8, device="cuda")
    sdgp.sdgp_residual_norm_backward(branch, out.detach(), torch.ones_like(branch), dy, post_weight=w["post"], gate=w["gate"], pre_weight=w["pre"],
                                     post_rstd=pr, pre_rstd=qr, alpha=ALPHA, n=n, m=m, seed=seed, values=vals, meta=meta, workspace=ws, **got)
    dh = torch.empty(rows, H, dtype=torch.bfloat16, device="cuda")
    sdgp.sdgp_spmm_linear(vals, meta, w["down"], dh)
    assert torch.equal(h.grad, dh) and torch.equal(x.grad, got["d_residual"]) and torch.equal(b["down"].grad, got["d_branch"].t() @ h.detach())
    for k in ("post", "pre"):
        assert torch.equal(b[k].grad, got["d_%s_weight" % k].bfloat16())
    assert torch.equal(b["gate"].grad, got["d_gate"].bfloat16())


def test_eight_bit_forward_with_the_pruned_backward():
    g = torch.Generator().manual_seed(5)
    x = torch.randn(3, 50, 256, generator=g).bfloat16().cuda().requires_grad_()
    w = (torch.randn(192, 256, generator=g) / 16).bfloat16().cuda().requires_grad_()
    d = torch.randn(3, 50, 192, generator=g).bfloat16().cuda()
    q, s = sdgp_fp8_weights(w)
    y = sdgp_linear_fp8(x, w)
    again = sdgp_linear_fp8(x, w, (q, s))
    assert torch.equal(y, again) and y.shape == (3, 50, 192)
    # each factor is off by 2^-4 of itself, or by half the smallest step: 2^-10 scales, and a scale is below max / 224
    size = x.detach().double().abs() @ w.detach().double().abs().t()
    small = 256 * (x.detach().abs().max() * w.detach().abs().max()).double() * 2 ** -10 / 224 * 2
    assert torch.all((y.double() - x.detach().double() @ w.detach().double().t()).abs() <= size * (2 ** -3 + 2 ** -7) + small)
    y.backward(d)
    x2, w2 = x.detach().clone().requires_grad_(), w.detach().clone().requires_grad_()
    sdgp_linear(x2, w2).backward(d)
    assert torch.equal(x.grad, x2.grad) and torch.equal(w.grad, w2.grad)


@pytest.mark.parametrize("fp8,n,m", [(False, 2, 4), (False, 1, 8), (True, 2, 4), (True, 1, 16), (True, 3, 4)])   # (sdgp_linear keeps two of a group at most)
def test_a_training_step_runs(fp8, n, m):
    blocks, head = parameters(128, 256, 192, 2, 3, torch.bfloat16, 6)   # (192 tokens: no compressed head, its dL/dO is pruned in a pass of its own)
    x = torch.randn(30, 128, device="cuda").bfloat16().requires_grad_()
    t = torch.randint(0, 190, (30,), device="cuda")
    lp, H = network(x, t, blocks, head, 190, n, m, fp8)
    (-lp.mean() + 0.01 * H.mean()).backward()
    for v in [x, head] + [v for b in blocks for v in b.values()]:
        assert torch.isfinite(v.grad).all() and v.grad.abs().max() > 0
    assert torch.all(head.grad[190:] == 0)


def test_a_captured_step_gives_the_eager_one():
    blocks, head = parameters(128, 128, 128, 1, 1, torch.bfloat16, 8)
    leaves = [head] + list(blocks[0].values())
    x = torch.randn(16, 128, device="cuda").bfloat16()
    t = torch.randint(0, 128, (16,), device="cuda")

    def step():
        lp, H = network(x, t, blocks, head, 128, 2, 4, True)
        return torch.autograd.grad(-lp.mean() + 0.1 * H.mean(), leaves)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            want = [v.clone() for v in step()]
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_parts_that_are_left_out():
    """No norms at all, gradients through one output only, no gradient asked for."""
    g = torch.Generator().manual_seed(9)
    x, r = (torch.randn(2, 20, 128, generator=g).bfloat16().cuda().requires_grad_() for _ in range(2))
    w = (torch.randn(128, 128, generator=g) / 11).bfloat16().cuda().requires_grad_()
    pre = torch.ones(128, device="cuda").bfloat16().requires_grad_()
    out, y = sdgp_linear_residual_norm(x, w, r, alpha=0.5, n=4, m=4)
    assert y is None and out.shape == r.shape
    out.sum().backward()
    assert torch.all(r.grad == 0.5)
    out, y = sdgp_linear_residual_norm(x, w, r, pre_weight=pre, n=4, m=4)
    out.float().square().sum().backward()          # nothing arrives at y
    assert torch.all(pre.grad == 0)
    with torch.no_grad():
        sdgp_linear_logprob(x, w, torch.zeros(2, 20, dtype=torch.int64, device="cuda"))
    lp, H = sdgp_linear_logprob(x.detach(), w, torch.zeros(2, 20, dtype=torch.int64, device="cuda"))
    H.sum().backward()
    assert lp.shape == (2, 20) and torch.isfinite(w.grad).all()
