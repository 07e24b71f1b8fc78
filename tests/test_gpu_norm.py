"""The boundary between two blocks (norms, gate, residual scale) and its gradient against their definitions in 64 bits.

Tolerances. Outputs are rounded once to their type: half a step, eps / 2 of the value. What comes before is fp32: a row's sums add 8
terms in a thread and 10 levels of joins (wide rows: C / 1024 terms more), each addition off by 2^-24 of the sum of magnitudes; rsqrtf
2^-22; ten operations on an element 2^-24 each, of the largest of its terms. `n` below counts those steps, `size` is the sum of the
magnitudes of the terms that make a value. Sums over rows add up to `rows` terms in sequence."""
import pytest
import torch

import paper_2202_00774_b200 as sdgp
from paper_2202_00774_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {B.BF16: torch.bfloat16, B.FP16: torch.float16, B.FP32: torch.float32}
EPS, ALPHA = 1e-6, 0.75


def state(rows, C, groups, dtype, seed, post=True, pre=True, gate=True):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    t = TYPES[dtype]
    s = {"branch": r(rows, C).to(t), "residual": (2 * r(rows, C)).to(t), "d_out": r(rows, C).to(t), "d_y": r(rows, C).to(t) if pre else None,
         "post_weight": (1 + 0.2 * r(C)).to(t) if post else None, "pre_weight": (1 + 0.2 * r(C)).to(t) if pre else None,
         "gate": (0.5 + 0.25 * r(groups, C)).to(t) if gate else None}
    return {k: v.cuda() if v is not None else None for k, v in s.items()}


def forward(s, dtype, out=None):
    rows = s["branch"].shape[0]
    out = torch.full_like(s["branch"], 9.0) if out is None else out
    y = torch.full_like(s["branch"], 9.0) if s["pre_weight"] is not None else None
    f = [torch.full((rows,), 9.0, device="cuda") for _ in range(2)]
    sdgp.sdgp_residual_norm(s["branch"], s["residual"], out, y, post_weight=s["post_weight"], gate=s["gate"], pre_weight=s["pre_weight"],
                            alpha=ALPHA, eps=EPS, dtype=dtype, post_rstd=f[0] if s["post_weight"] is not None else None,
                            pre_rstd=f[1] if s["pre_weight"] is not None else None)
    return out, y, f[0], f[1]


def backward(s, dtype, out, post_rstd, pre_rstd, want=("d_residual", "d_branch", "d_gate", "d_post_weight", "d_pre_weight"), **more):
    b = s["branch"]
    rows, C = b.shape
    groups = 1 if s["gate"] is None else s["gate"].shape[0]
    got = {}
    for k in want:
        if k in ("d_residual", "d_branch"):
            got[k] = torch.full_like(b, 9.0)
        elif s[k[2:]] is not None:
            got[k] = torch.full(s[k[2:]].shape, 9.0, device="cuda")
    ws = torch.empty(sdgp.sdgp_workspace_size_residual_norm_backward(rows, C, groups), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)   # NaN wherever something is read that was not written
    sdgp.sdgp_residual_norm_backward(b, out, s["d_out"], s["d_y"], post_weight=s["post_weight"], gate=s["gate"], pre_weight=s["pre_weight"],
                                     post_rstd=post_rstd if s["post_weight"] is not None else None,
                                     pre_rstd=pre_rstd if s["d_y"] is not None else None, alpha=ALPHA, dtype=dtype, workspace=ws, **got, **more)
    return got


def d64(x):
    return None if x is None else x.double().cpu()


def definition(s):
    b, r, wp, g, w = (d64(s[k]) for k in ("branch", "residual", "post_weight", "gate", "pre_weight"))
    rows, C = b.shape
    post = pre = y = ysize = None
    n = b
    if wp is not None:
        post = (b.square().mean(1) + EPS) ** -0.5
        n = b * post[:, None] * wp
    g = torch.ones(1, C, dtype=torch.float64) if g is None else g
    g = g.repeat_interleave(rows // g.shape[0], 0)
    out = ALPHA * r + g * n
    size = (ALPHA * r).abs() + (g * n).abs()
    if w is not None:
        pre = (out.square().mean(1) + EPS) ** -0.5
        y, ysize = out * pre[:, None] * w, size * pre[:, None] * w.abs()
    return out, y, post, pre, size, ysize


def gradients(s, out, post_rstd, pre_rstd):
    """The gradients, and for each the sum of magnitudes that it is made of."""
    b, wp, gate, w, do, dy, o = (d64(x) for x in (s["branch"], s["post_weight"], s["gate"], s["pre_weight"], s["d_out"], s["d_y"], out))
    rows, C = b.shape
    g = torch.ones(1, C, dtype=torch.float64) if gate is None else gate
    groups = g.shape[0]
    g = g.repeat_interleave(rows // groups, 0)
    got, size = {}, {}
    d = torch.zeros_like(b) if do is None else do
    ds = d.abs()
    if dy is not None:
        k = d64(pre_rstd)[:, None]
        u, wd = o * k, dy * w
        m = (wd * u).mean(1, keepdim=True)
        d = d + k * (wd - u * m)
        ds = ds + k * (wd.abs() + u.abs() * (wd * u).abs().mean(1, keepdim=True))
        got["d_pre_weight"], size["d_pre_weight"] = (dy * u).sum(0), (dy * u).abs().sum(0)
    got["d_residual"], size["d_residual"] = ALPHA * d, ALPHA * ds
    v = b
    if wp is not None:
        k = d64(post_rstd)[:, None]
        v = b * k
        got["d_post_weight"], size["d_post_weight"] = (d * g * v).sum(0), (ds * (g * v).abs()).sum(0)
        q, qs = d * g * wp, ds * (g * wp).abs()
        got["d_branch"] = k * (q - v * (q * v).mean(1, keepdim=True))
        size["d_branch"] = k * (qs + v.abs() * (qs * v.abs()).mean(1, keepdim=True))
    else:
        got["d_branch"], size["d_branch"] = d * g, ds * g.abs()
    if gate is not None:
        n, ns = (d * v * (1 if wp is None else wp)), (ds * (v * (1 if wp is None else wp)).abs())
        got["d_gate"], size["d_gate"] = n.view(groups, -1, C).sum(1), ns.view(groups, -1, C).sum(1)
    return got, size


def near(x, want, size, dtype, n):
    fi = torch.finfo(TYPES[dtype]) if x.dtype != torch.float32 else torch.finfo(torch.float32)
    tol = n * 2 ** -24 * size + want.abs() * fi.eps / 2 + fi.smallest_normal * fi.eps
    off = (x.double().cpu() - want).abs()
    assert torch.all(off <= tol), ((off - tol).max(), off.max())


SHAPES = [(1, 1, 1), (2, 3, 1), (5, 8, 5), (7, 17, 1), (3, 64, 1), (33, 250, 1), (130, 256, 2), (64, 263, 8), (40, 1024, 40), (700, 520, 7),
          (19, 1999, 1), (24, 1999, 8), (1064, 1001, 8), (300, 2044, 300), (9, 4096, 1), (500, 4096, 2), (3, 8185, 3), (4, 8192, 1), (6, 8193, 2),
          (5, 16384, 1), (300, 12002, 3), (21, 1003, 7), (600, 99, 200), (2000, 36, 500), (3000, 40, 3000), (4001, 51, 4001),
          (300, 16383, 1), (7, 20000, 1), (200, 24000, 2), (40, 32761, 1), (9, 40000, 3),
          # more gates than groups of threads, for every number of threads that a row may have
          (5000, 500, 5000), (3000, 1000, 3000), (1500, 2000, 1500), (700, 4000, 700), (400, 8000, 400), (300, 9001, 300), (1500, 1999, 1500),
          (900, 7999, 300), (6000, 333, 3000), (1200, 4001, 400)]


@pytest.mark.parametrize("dtype", [B.BF16, B.FP16, B.FP32])
@pytest.mark.parametrize("rows,C,groups", SHAPES)
def test_forward_and_gradient(dtype, rows, C, groups):
    for post, pre, gate in ((True, True, True), (False, True, True), (True, False, False)) if rows * C < 10000 else ((True, True, True),):
        s = state(rows, C, groups if gate else 1, dtype, rows + C, post, pre, gate)
        out, y, post_rstd, pre_rstd = forward(s, dtype)
        want = definition(s)
        n = 40 + C / 1024
        near(out, want[0], want[4], dtype, n)
        if pre:
            near(y, want[1], want[5], dtype, n)
            near(pre_rstd, want[3], want[3], B.FP32, n)
        if post:
            near(post_rstd, want[2], want[2], B.FP32, n)
        got = backward(s, dtype, out, post_rstd, pre_rstd)
        ref, size = gradients(s, out, post_rstd, pre_rstd)
        assert sorted(got) == sorted(ref)
        for k in ref:
            near(got[k], ref[k], size[k], dtype, 2 * n + (rows if got[k].dtype == torch.float32 and k not in ("d_branch", "d_residual") else 0))


@pytest.mark.parametrize("C", [96, 513, 9000])
def test_gradients_one_at_a_time(C):
    """Each output alone, no gradient on the stream, none at y; and in the place of an input."""
    s = state(50, C, 5, B.BF16, 3)
    out, y, post_rstd, pre_rstd = forward(s, B.BF16)
    everything = backward(s, B.BF16, out, post_rstd, pre_rstd)
    for k in everything:
        one = backward(s, B.BF16, out, post_rstd, pre_rstd, want=(k,))
        assert torch.equal(one[k], everything[k]), k
    for missing in ("d_out", "d_y"):
        t = {**s, missing: None}
        got = backward(t, B.BF16, out, post_rstd, pre_rstd, want=("d_residual", "d_branch", "d_gate", "d_post_weight"))
        ref, size = gradients(t, out, post_rstd, pre_rstd)
        for k in got:
            near(got[k], ref[k], size[k], B.BF16, 100 + 50)
    r = s["residual"].clone()
    got = forward({**s, "residual": r}, B.BF16, out=r)
    assert got[0] is r and torch.equal(r, out) and torch.equal(got[1], y)
    d = s["d_out"].clone()
    ws = torch.empty(sdgp.sdgp_workspace_size_residual_norm_backward(50, C, 5), dtype=torch.uint8, device="cuda")
    sdgp.sdgp_residual_norm_backward(s["branch"], out, d, s["d_y"], post_weight=s["post_weight"], gate=s["gate"], pre_weight=s["pre_weight"],
                                     post_rstd=post_rstd, pre_rstd=pre_rstd, alpha=ALPHA, d_residual=d, workspace=ws)
    assert torch.equal(d, everything["d_residual"])


def test_gradient_against_differences():
    s = state(3, 11, 1, B.FP32, 5)
    out, _, post_rstd, pre_rstd = forward(s, B.FP32)
    got = backward(s, B.FP32, out, post_rstd, pre_rstd)

    def value(t):
        o, y = definition(t)[:2]
        return ((o * d64(s["d_out"])).sum() + (y * d64(s["d_y"])).sum()).item()

    step = 2.0 ** -12
    for name, key in (("branch", "d_branch"), ("residual", "d_residual"), ("gate", "d_gate"), ("post_weight", "d_post_weight"), ("pre_weight", "d_pre_weight")):
        for i in (0, 7):
            up, down = s[name].double().clone(), s[name].double().clone()
            up.view(-1)[i] += step
            down.view(-1)[i] -= step
            slope = (value({**s, name: up}) - value({**s, name: down})) / (2 * step)
            # step^2 / 6 times a third derivative of at most some hundreds
            assert abs(got[key].view(-1)[i].item() - slope) <= 1e3 * step ** 2 + 1e-5 * (1 + abs(slope)), (name, i)


@pytest.mark.parametrize("dtype", [B.BF16, B.FP16])
@pytest.mark.parametrize("n,m", [(1, 4), (2, 4), (1, 8), (2, 8), (1, 16), (2, 16), (1, 32), (2, 32)])
def test_pruned_copy_is_algorithm_1_on_the_gradient(dtype, n, m):
    for rows, C in ((5, 96), (70, 1056), (3, 9216)):
        s = state(rows, C, 1, dtype, n * m)
        out, _, post_rstd, pre_rstd = forward(s, dtype)
        for scheme in (B.RANDOM, B.MAGNITUDE, B.RESCALED_MAGNITUDE):
            pairs = [(torch.zeros(rows, C // 2, dtype=out.dtype, device="cuda"), torch.zeros(rows, C // 16, dtype=torch.int16, device="cuda")) for _ in range(3)]
            more = dict(n=n, m=m, scheme=scheme, seed=1234567)
            got = backward(s, dtype, out, post_rstd, pre_rstd, values=pairs[0][0], meta=pairs[0][1], **more)
            backward(s, dtype, out, post_rstd, pre_rstd, want=(), values=pairs[1][0], meta=pairs[1][1], **more)
            sdgp.sdgp_prune_typed(got["d_branch"], n, m, scheme, 1234567, dtype, values=pairs[2][0], meta=pairs[2][1])
            for v, e in pairs[:2]:
                assert torch.equal(v.view(torch.int16), pairs[2][0].view(torch.int16)) and torch.equal(e, pairs[2][1])


def test_sums_do_not_depend_on_the_run():
    s = state(3000, 1000, 4, B.BF16, 6)
    out, _, post_rstd, pre_rstd = forward(s, B.BF16)
    first = backward(s, B.BF16, out, post_rstd, pre_rstd)
    for _ in range(3):
        again = backward(s, B.BF16, out, post_rstd, pre_rstd)
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_numbers_that_are_not_finite_stay_in_their_row():
    s = state(6, 500, 1, B.BF16, 7)
    s["branch"][1, 3], s["branch"][3, 499], s["residual"][4, 0] = float("nan"), float("inf"), float("nan")
    out, y, post_rstd, pre_rstd = forward(s, B.BF16)
    for r in (0, 2, 5):
        assert torch.isfinite(out[r]).all() and torch.isfinite(y[r]).all()
    for r in (1, 3, 4):
        assert torch.isnan(y[r]).any()


def test_streams_and_graphs():
    s = state(64, 768, 8, B.BF16, 8)
    out, y, post_rstd, pre_rstd = forward(s, B.BF16)
    want = backward(s, B.BF16, out, post_rstd, pre_rstd)
    got = {k: torch.zeros_like(v) for k, v in want.items()}
    o2, y2, a2, b2 = torch.zeros_like(out), torch.zeros_like(y), torch.zeros_like(post_rstd), torch.zeros_like(pre_rstd)
    ws = torch.empty(sdgp.sdgp_workspace_size_residual_norm_backward(64, 768, 8), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        sdgp.sdgp_residual_norm(s["branch"], s["residual"], o2, y2, post_weight=s["post_weight"], gate=s["gate"], pre_weight=s["pre_weight"],
                                alpha=ALPHA, eps=EPS, post_rstd=a2, pre_rstd=b2)
        sdgp.sdgp_residual_norm_backward(s["branch"], o2, s["d_out"], s["d_y"], post_weight=s["post_weight"], gate=s["gate"],
                                         pre_weight=s["pre_weight"], post_rstd=a2, pre_rstd=b2, alpha=ALPHA, workspace=ws, **got)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o2, out) and torch.equal(y2, y) and all(torch.equal(got[k], want[k]) for k in want)


def test_the_sum_in_the_branchs_place():
    for C in (256, 1001, 20000):
        s = state(40, C, 1, B.BF16, 11)
        out, y, post_rstd, pre_rstd = forward(s, B.BF16)
        b = s["branch"].clone()
        got = forward({**s, "branch": b}, B.BF16, out=b)
        assert torch.equal(b, out) and torch.equal(got[1], y)


def test_two_streams_at_once():
    s = [state(500, 1999, 4, B.BF16, k) for k in (12, 13)]
    want = []
    for k in range(2):
        f = forward(s[k], B.BF16)
        want.append((f, backward(s[k], B.BF16, f[0], f[2], f[3])))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                f = forward(s[k], B.BF16)
                got[k].append((f, backward(s[k], B.BF16, f[0], f[2], f[3])))
    torch.cuda.synchronize()
    for k in range(2):
        for f, g in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(f, want[k][0])) and all(torch.equal(g[n], want[k][1][n]) for n in g)


@pytest.mark.parametrize("dtype", [B.BF16, B.FP32])
@pytest.mark.parametrize("rows,C", [(300, 9000), (500, 16384), (261, 12007), (150, 32760), (1, 16384)])
def test_rows_of_several_ctas_repeat_themselves(dtype, rows, C):
    """Rows that a cluster shares: every call gives the same bits, also with two streams at work, and no wait runs out."""
    s = state(rows, C, 1, dtype, C + rows)
    f = forward(s, dtype)
    want = backward(s, dtype, f[0], f[2], f[3])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(20):
        with torch.cuda.stream(streams[i % 2]):
            got.append(backward(s, dtype, f[0], f[2], f[3]))
    torch.cuda.synchronize()
    assert all(torch.equal(g[n], want[n]) for g in got for n in g)
    assert sdgp.sdgp_last_device_error() == 0


def test_no_rows():
    s = state(0, 64, 1, B.BF16, 9)
    g = {k: torch.full(sh, 5.0, device="cuda") for k, sh in (("d_gate", (1, 64)), ("d_post_weight", (64,)), ("d_pre_weight", (64,)))}
    f = torch.empty(0, device="cuda")
    sdgp.sdgp_residual_norm(s["branch"], s["residual"], s["branch"], s["branch"], pre_weight=s["pre_weight"])
    sdgp.sdgp_residual_norm_backward(s["branch"], s["branch"], s["d_out"], s["d_y"], post_weight=s["post_weight"], gate=s["gate"],
                                     pre_weight=s["pre_weight"], post_rstd=f, pre_rstd=f, **g)
    assert all((v == 0).all() for v in g.values())


def test_calls_that_are_refused():
    s = state(4, 64, 1, B.BF16, 1)
    o = torch.empty_like(s["branch"])
    with pytest.raises(ValueError):
        sdgp.sdgp_residual_norm(s["branch"], s["residual"][:3], o)
    with pytest.raises(ValueError):
        sdgp.sdgp_residual_norm(s["branch"], s["residual"], o, dtype=B.FP32)
    with pytest.raises(ValueError):
        sdgp.sdgp_residual_norm(s["branch"], s["residual"], o, gate=torch.ones(100, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(sdgp.SdgpError):   # three gates for four rows
        sdgp.sdgp_residual_norm(s["branch"], s["residual"], o, gate=torch.ones(3, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(sdgp.SdgpError):   # y without its weight
        sdgp.sdgp_residual_norm(s["branch"], s["residual"], o, o)
    with pytest.raises(sdgp.SdgpError):   # no workspace
        sdgp.sdgp_residual_norm_backward(s["branch"], None, s["d_out"], d_residual=o)
