"""What the language-model operators of this library are measured on: the cases, their inputs, the calls and the plain forms.

A network of linear layers whose data gradient is pruned (``sdgp_linear``) needs, as a language model, what stands between
those layers and at their end: the norms around a block with its residual sum, gate and residual scale; the log
probabilities of the tokens (whose gradient is the first dL/dO that is pruned); and, where the forward product runs in
8 bits, the quantisation to e4m3 with a scale for each block of 128 and the product of two such matrices.

``own`` false: elementary torch operations in 32 bits (indices and selections exact), rounded once at the end.
``own`` true: the calls a training or serving loop makes through the public entry points. ``exact`` states the same
results in 64 bits from the definitions.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
CODES = {"bf16": 0, "fp16": 1, "fp32": 2}   # sdgp_dtype
BLOCK = 128        # elements of a row that share one scale
E4M3_MAX = 448.0
EPS = 1e-6


# ------------------------------------------------------------------ cases


def listed():
    return [
        # one generated token of a served model: its 20 best alternatives beside its log probability; latency
        {"name": "logprob_token", "op": "logprob", "rows": 1, "width": 131072, "classes": 131072, "dtype": "bf16", "top": 20},
        # the head of a training step; a vocabulary padded to whole blocks of 64 output features
        {"name": "logprob_step", "op": "logprob", "rows": 4096, "width": 50048, "classes": 50001, "dtype": "fp16", "top": 0},
        # gradient of the loss with an entropy bonus, the largest head
        {"name": "logprob_backward_step", "op": "logprob_backward", "rows": 4096, "width": 131072, "classes": 131072,
         "dtype": "bf16", "entropy": True},
        # a short batch against fp32 logits of a vocabulary of odd length
        {"name": "logprob_backward_odd", "op": "logprob_backward", "rows": 333, "width": 32003, "classes": 32003,
         "dtype": "fp32", "entropy": False},
        # a served model's block boundary for one token; latency
        {"name": "norm_token", "op": "norm", "rows": 1, "width": 4096, "groups": 1, "post": True, "pre": True, "dtype": "bf16"},
        # the block boundary of a training step: 8 sequences of 2048 tokens
        {"name": "norm_step", "op": "norm", "rows": 16384, "width": 4096, "groups": 1, "post": True, "pre": True, "dtype": "bf16"},
        # its gradient
        {"name": "norm_backward_step", "op": "norm_backward", "rows": 16384, "width": 4096, "groups": 1, "post": True,
         "pre": True, "dtype": "bf16"},
        # a width that is no multiple of anything, one gate for each of eight sequences (a gate that depends on a condition)
        {"name": "norm_backward_odd", "op": "norm_backward", "rows": 1064, "width": 1999, "groups": 8, "post": True,
         "pre": True, "dtype": "fp16"},
        # activations before an 8-bit product: a scale for each row and 128 columns
        {"name": "quantize_activations", "op": "quantize", "rows": 16384, "width": 4096, "block_rows": 1, "dtype": "bf16"},
        # fp32 master weights: a scale for each 128 x 128 block
        {"name": "quantize_weights", "op": "quantize", "rows": 2112, "width": 2688, "block_rows": 128, "dtype": "fp32"},
        # a linear layer for one generated token: the weights are read once
        {"name": "fp8_linear_token", "op": "fp8_linear", "rows": 1, "features": 4096, "width": 4096, "dtype": "bf16"},
        # the large fully connected layer of the benchmark, forward
        {"name": "fp8_linear_step", "op": "fp8_linear", "rows": 16384, "features": 4096, "width": 4096, "dtype": "bf16"},
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(["logprob", "logprob_backward", "norm", "norm_backward", "quantize", "fp8_linear"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("logprob", "logprob_backward"):
        width = _log_uniform(rng, 64, 262144)
        if rng.random() < 0.6:   # what sdgp_linear makes: a multiple of 64
            width = (width + 63) // 64 * 64
        classes = width - (rng.randrange(0, 64) if width > 128 and rng.random() < 0.5 else 0)
        rows = _log_uniform(rng, 1, min(16384, (1 << 28) // width))
        case = {"op": op, "rows": rows, "width": width, "classes": classes, "dtype": dtype}
        if op == "logprob":
            return {**case, "top": min(rng.choice([0, 0, 1, 5, 20, 32]), classes)}
        return {**case, "entropy": rng.random() < 0.5}
    if op in ("norm", "norm_backward"):
        width = _log_uniform(rng, 32, 16384)
        if rng.random() < 0.7:
            width = (width + 63) // 64 * 64
        rows = _log_uniform(rng, 1, min(16384, (1 << 26) // width))
        groups = rng.choice([1, 1, rows, 8])
        if groups == 8:   # eight sequences
            rows = (rows + 7) // 8 * 8
        post, pre = rng.choice([(True, True), (True, True), (True, False), (False, True)])
        return {"op": op, "rows": rows, "width": width, "groups": groups, "post": post, "pre": pre, "dtype": dtype}
    if op == "quantize":
        width = _log_uniform(rng, 16, 16384) // 16 * 16
        return {"op": op, "rows": _log_uniform(rng, 1, min(16384, (1 << 26) // width)), "width": width,
                "block_rows": rng.choice([1, 128]), "dtype": dtype}
    width = _log_uniform(rng, 128, 8192) // 16 * 16
    features = _log_uniform(rng, 64, 8192)
    if rng.random() < 0.8:
        features = (features + 7) // 8 * 8
    return {"op": op, "rows": _log_uniform(rng, 1, 8192), "features": features, "width": width, "dtype": dtype}


# ------------------------------------------------------------------ inputs


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _scales(x, block_rows):
    """The power of two s of each block of `block_rows` x 128 for which max|x| / s lies in (224, 448]; 1 for a block of zeros."""
    rows, width = x.shape
    down, right = -rows % block_rows, -width % BLOCK
    blocks = torch.nn.functional.pad(x.float().abs(), (0, right, 0, down))
    most = blocks.view((rows + down) // block_rows, block_rows, (width + right) // BLOCK, BLOCK).amax((1, 3))
    mantissa, exponent = torch.frexp(most)   # most = mantissa 2^exponent, mantissa in [1/2, 1); 448 = 0.875 * 2^9
    exponent = torch.where(mantissa > 0.875, exponent - 8, exponent - 9).clamp(min=-126)
    power = ((exponent + 127) << 23).view(torch.float32)   # 2^exponent, put together from its bits
    return torch.where(most > 0, power, torch.ones_like(most))


def _spread(scales, block_rows, rows, width):
    """The scale of every element."""
    return scales.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :width]


def _quantize(x, block_rows):
    s = _scales(x, block_rows)
    return (x.float() / _spread(s, block_rows, *x.shape)).to(torch.float8_e4m3fn), s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    s = dict(case)
    op, rows, width = case["op"], case["rows"], case["width"]
    if op in ("logprob", "logprob_backward"):
        classes = case["classes"]
        logits = _normal(g, rows, width).mul_(2.5)
        targets = torch.randint(0, classes, (rows,), generator=g, device="cuda")
        sure = torch.rand(rows, generator=g, device="cuda") < 0.6   # tokens that the model expects
        boost = torch.where(sure, 8.0 + 6.0 * torch.rand(rows, generator=g, device="cuda"), torch.zeros((), device="cuda"))
        logits.scatter_add_(1, targets[:, None], boost[:, None])
        targets[torch.rand(rows, generator=g, device="cuda") < 0.05] = -100   # padding: tokens that are not counted
        s["logits"], s["targets"] = logits.to(dtype), targets
        if op == "logprob_backward":   # what the forward pass has left, and the gradients of what it gave
            x = s["logits"][:, :classes].float()
            s["lse"] = torch.logsumexp(x, 1)
            logp = x.sub_(s["lse"][:, None])
            s["entropy_of_row"] = -torch.einsum("rc,rc->r", logp.exp(), logp) if case["entropy"] else None
            s["d_logprob"] = -(0.5 + torch.rand(rows, generator=g, device="cuda")) / rows
            s["d_entropy"] = _normal(g, rows).mul_(0.1 / rows) if case["entropy"] else None
        return s
    if op in ("norm", "norm_backward"):
        s["branch"] = _normal(g, rows, width).to(dtype)
        residual = (_normal(g, rows, width) * 2.0).to(dtype)
        s["post_weight"] = (1.0 + 0.2 * _normal(g, width)).to(dtype) if case["post"] else None
        s["pre_weight"] = (1.0 + 0.2 * _normal(g, width)).to(dtype) if case["pre"] else None
        s["gate"] = (0.5 + 0.25 * _normal(g, case["groups"], width)).to(dtype)
        s["alpha"] = 0.75
        if op == "norm":
            s["residual"] = residual
            return s
        out, _, post_rstd, pre_rstd = _norm_plain({**s, "residual": residual})
        s["out"], s["post_rstd"], s["pre_rstd"] = out, post_rstd, pre_rstd
        s["d_out"] = _normal(g, rows, width).to(dtype)
        s["d_y"] = _normal(g, rows, width).to(dtype) if case["pre"] else None
        return s
    if op == "quantize":
        x = _normal(g, rows, width)
        if case["block_rows"] == 1:   # a few channels of an activation are far larger than the others
            x.mul_(torch.where(torch.rand(width, generator=g, device="cuda") < 0.01, 20.0, 1.0))
        s["x"] = x.to(dtype)
        return s
    s["xq"], s["x_scale"] = _quantize(_normal(g, rows, width), 1)
    # weights with the scales of a checkpoint: any positive number, not powers of two alone
    s["wq"], w_scale = _quantize(_normal(g, case["features"], width) / math.sqrt(width), BLOCK)
    s["w_scale"] = w_scale * (0.75 + 0.5 * torch.rand(w_scale.shape, generator=g, device="cuda"))
    return s


# ------------------------------------------------------------------ plain forms


def _logprob_plain(s):
    x = s["logits"][:, :s["classes"]].float()
    most = x.amax(1)
    lse = (x - most[:, None]).exp().sum(1).log() + most
    counted = s["targets"] >= 0
    logprob = torch.where(counted, x.gather(1, s["targets"].clamp(min=0)[:, None])[:, 0] - lse, 0.0)
    out = {"logprob": logprob, "lse": lse}
    logp = x - lse[:, None]
    out["entropy"] = -(logp.exp() * logp).sum(1)
    if s["top"]:
        # the largest first, equal ones by their index: one whole number that orders both, and no two alike
        bits = (s["logits"][:, :s["classes"]].float() + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = order * (1 << 32) + (0xFFFFFFFF - torch.arange(s["classes"], device=x.device))
        out["top_token"] = 0xFFFFFFFF - (key.topk(s["top"], dim=1).values & 0xFFFFFFFF)
        out["top_logprob"] = logp.gather(1, out["top_token"])
    return out


def _logprob_backward_plain(s):
    logits, classes = s["logits"], s["classes"]
    logp = logits[:, :classes].float() - s["lse"][:, None]
    counted = s["targets"] >= 0
    d = torch.where(counted, s["d_logprob"], 0.0)
    factor = d[:, None]
    if s["entropy"]:
        factor = factor + s["d_entropy"][:, None] * (logp + s["entropy_of_row"][:, None])
    grad = torch.zeros(logits.shape, device=logits.device)
    grad[:, :classes] = -(logp.exp() * factor)
    grad.scatter_add_(1, s["targets"].clamp(min=0)[:, None], d[:, None])
    return grad.to(logits.dtype)


def _norm_plain(s):
    b, r = s["branch"].float(), s["residual"].float()
    rows, width = b.shape
    post_rstd = pre_rstd = y = None
    n = b
    if s["post"]:
        post_rstd = torch.rsqrt((b * b).mean(1) + EPS)
        n = b * post_rstd[:, None] * s["post_weight"].float()
    gate = s["gate"].float()
    out = s["alpha"] * r + (gate[:, None, :] * n.view(gate.shape[0], -1, width)).view(rows, width)
    if s["pre"]:
        pre_rstd = torch.rsqrt((out * out).mean(1) + EPS)
        y = (out * pre_rstd[:, None] * s["pre_weight"].float()).to(s["branch"].dtype)
    return out.to(s["branch"].dtype), y, post_rstd, pre_rstd


def _norm_backward_plain(s):
    dtype = s["branch"].dtype
    b, d = s["branch"].float(), s["d_out"].float()
    rows, width = b.shape
    got = {}
    if s["pre"]:
        unit = s["out"].float() * s["pre_rstd"][:, None]
        dy = s["d_y"].float()
        wd = dy * s["pre_weight"].float()
        d = d + s["pre_rstd"][:, None] * (wd - unit * (wd * unit).mean(1, keepdim=True))
        got["d_pre_weight"] = (dy * unit).sum(0)
    got["d_residual"] = (s["alpha"] * d).to(dtype)
    gate = s["gate"].float()
    unit = b * s["post_rstd"][:, None] if s["post"] else b
    n = unit * s["post_weight"].float() if s["post"] else unit
    got["d_gate"] = (d * n).view(gate.shape[0], -1, width).sum(1)
    dn = (d.view(gate.shape[0], -1, width) * gate[:, None, :]).view(rows, width)
    if s["post"]:
        got["d_post_weight"] = (dn * unit).sum(0)
        wd = dn * s["post_weight"].float()
        dn = s["post_rstd"][:, None] * (wd - unit * (wd * unit).mean(1, keepdim=True))
    got["d_branch"] = dn.to(dtype)
    return got


def _fp8_linear_plain(s):
    x = s["xq"].float() * _spread(s["x_scale"], 1, *s["xq"].shape)
    w = s["wq"].float() * _spread(s["w_scale"], BLOCK, *s["wq"].shape)
    return (x @ w.t()).to(TYPES[s["dtype"]])


# ------------------------------------------------------------------ the measured calls


def run(state):
    s = state
    op = s["op"]
    if own:
        return _run_own(s)
    if op == "logprob":
        return _logprob_plain(s)
    if op == "logprob_backward":
        return _logprob_backward_plain(s)
    if op == "norm":
        return _norm_plain(s)
    if op == "norm_backward":
        return _norm_backward_plain(s)
    if op == "quantize":
        q, scale = _quantize(s["x"], s["block_rows"])
        return {"values": q.bfloat16(), "scale": scale}   # what is held in 8 bits, as the values it stands for (exact in bf16)
    return _fp8_linear_plain(s)


def _run_own(s):
    import paper_2202_00774_b200 as sdgp
    op, rows, code = s["op"], s["rows"], CODES[s["dtype"]]
    if op == "logprob":
        logits, top = s["logits"], s["top"]
        f32 = dict(dtype=torch.float32, device=logits.device)
        out = {k: torch.empty(rows, **f32) for k in ("logprob", "lse", "entropy")}
        if top:
            out["top_token"] = torch.empty(rows, top, dtype=torch.int64, device=logits.device)
            out["top_logprob"] = torch.empty(rows, top, **f32)
        sdgp.sdgp_token_logprob(logits, s["targets"], classes=s["classes"], dtype=code, **out)
        return out
    if op == "logprob_backward":
        grad = torch.empty_like(s["logits"])
        sdgp.sdgp_token_logprob_backward(s["logits"], s["targets"], s["lse"], s["d_logprob"], grad=grad, classes=s["classes"],
                                         dtype=code, entropy=s["entropy_of_row"], d_entropy=s["d_entropy"])
        return grad
    if op == "norm":
        b = s["branch"]
        out = torch.empty_like(b)
        y = torch.empty_like(b) if s["pre"] else None
        post_rstd = torch.empty(rows, device=b.device) if s["post"] else None
        pre_rstd = torch.empty(rows, device=b.device) if s["pre"] else None
        sdgp.sdgp_residual_norm(b, s["residual"], out, y, post_weight=s["post_weight"], gate=s["gate"],
                                pre_weight=s["pre_weight"], alpha=s["alpha"], eps=EPS, dtype=code, post_rstd=post_rstd,
                                pre_rstd=pre_rstd)
        return out, y, post_rstd, pre_rstd
    if op == "norm_backward":
        b = s["branch"]
        f32 = dict(dtype=torch.float32, device=b.device)
        got = {"d_residual": torch.empty_like(b), "d_branch": torch.empty_like(b),
               "d_gate": torch.empty(s["gate"].shape, **f32)}
        if s["post"]:
            got["d_post_weight"] = torch.empty(s["width"], **f32)
        if s["pre"]:
            got["d_pre_weight"] = torch.empty(s["width"], **f32)
        need = sdgp.sdgp_workspace_size_residual_norm_backward(rows, s["width"], s["gate"].shape[0])
        workspace = torch.empty(max(16, need), dtype=torch.uint8, device=b.device)
        sdgp.sdgp_residual_norm_backward(b, s["out"], s["d_out"], s["d_y"], post_weight=s["post_weight"], gate=s["gate"],
                                         pre_weight=s["pre_weight"], post_rstd=s["post_rstd"], pre_rstd=s["pre_rstd"],
                                         alpha=s["alpha"], dtype=code, workspace=workspace, **got)
        return got
    if op == "quantize":
        x = s["x"]
        q = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=x.device)
        scale = torch.empty(-(-rows // s["block_rows"]), -(-s["width"] // BLOCK), device=x.device)
        sdgp.sdgp_fp8_quantize(x, q, scale, block_rows=s["block_rows"], dtype=code)
        return {"values": q.bfloat16(), "scale": scale}
    y = torch.empty(rows, s["features"], dtype=TYPES[s["dtype"]], device=s["xq"].device)
    sdgp.sdgp_fp8_linear(s["xq"], s["x_scale"], s["wq"], s["w_scale"], y, dtype=code)
    return y


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    op, rows, width = case["op"], case["rows"], case["width"]
    if op == "logprob":
        # logits and targets in; three numbers a row and the alternatives out; per logit: difference, exp, two sums
        return {"bytes": rows * (case["classes"] * size + 8 + 12 + case["top"] * 12), "flops": rows * case["classes"] * 5}
    if op == "logprob_backward":
        # logits in (the padding is not looked at), the whole gradient out
        return {"bytes": rows * ((case["classes"] + width) * size + 8 + (16 if case["entropy"] else 8)),
                "flops": rows * case["classes"] * (5 if case["entropy"] else 3)}
    if op == "norm":
        tensors = 3 + (1 if case["pre"] else 0)
        vectors = case["groups"] + (1 if case["post"] else 0) + (1 if case["pre"] else 0)
        return {"bytes": size * width * (rows * tensors + vectors) + 4 * rows * ((1 if case["post"] else 0) + (1 if case["pre"] else 0)),
                "flops": rows * width * (3 + (4 if case["post"] else 0) + (4 if case["pre"] else 0))}
    if op == "norm_backward":
        tensors = 4 + (2 if case["pre"] else 0)
        vectors = case["groups"] + (1 if case["post"] else 0) + (1 if case["pre"] else 0)
        return {"bytes": size * width * (rows * tensors + vectors) + 4 * width * vectors
                + 4 * rows * ((1 if case["post"] else 0) + (1 if case["pre"] else 0)),
                "flops": rows * width * (4 + (9 if case["post"] else 0) + (9 if case["pre"] else 0))}
    blocks = -(-width // BLOCK)
    if op == "quantize":
        return {"bytes": rows * width * (size + 1) + 4 * blocks * -(-rows // case["block_rows"]), "flops": rows * width * 2}
    features = case["features"]
    return {"bytes": (rows + features) * width + 4 * blocks * (rows + -(-features // BLOCK)) + rows * features * size,
            "flops": 2 * rows * features * width}


# ------------------------------------------------------------------ the definitions, in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    op, rows, width = case["op"], case["rows"], case["width"]
    if op == "logprob":
        found = {"logprob": [], "lse": [], "entropy": []}
        if case["top"]:
            found["top_logprob"] = []
        step = max(1, (1 << 27) // width)
        for i in range(0, rows, step):   # in pieces: 64-bit copies of the largest logits are large
            z = s["logits"][i:i + step, :case["classes"]].double()
            t = s["targets"][i:i + step]
            lse = torch.logsumexp(z, dim=1)
            p = torch.exp(z - lse[:, None])
            own_logit = z[torch.arange(len(t), device=z.device), t.clamp(min=0)]
            found["logprob"].append(torch.where(t < 0, torch.zeros_like(lse), own_logit - lse))
            found["lse"].append(lse)
            found["entropy"].append(lse - (p * z).sum(dim=1))
            if case["top"]:
                found["top_logprob"].append(torch.topk(z, case["top"], dim=1)[0] - lse[:, None])
        got = {k: torch.cat(v) for k, v in found.items()}
        return {**got, "top_token": None} if case["top"] else got
    if op == "logprob_backward":
        grad = torch.zeros(rows, width, dtype=torch.float64, device="cuda")
        step = max(1, (1 << 27) // width)
        for i in range(0, rows, step):
            z = s["logits"][i:i + step, :case["classes"]].double()
            t = s["targets"][i:i + step]
            lse = s["lse"][i:i + step].double()[:, None]
            p = torch.exp(z - lse)
            hot = torch.zeros_like(z)
            hot[torch.arange(len(t), device=z.device), t.clamp(min=0)] = 1.0
            # d logprob / d z = onehot - p; d entropy / d z = -p (log p + H)
            part = (s["d_logprob"][i:i + step].double() * (t >= 0))[:, None] * (hot - p)
            if case["entropy"]:
                part -= s["d_entropy"][i:i + step].double()[:, None] * p * (z - lse + s["entropy_of_row"][i:i + step].double()[:, None])
            grad[i:i + step, :case["classes"]] = part
        return grad
    if op == "norm":
        b, r = s["branch"].double(), s["residual"].double()
        gate = s["gate"].double().repeat_interleave(rows // case["groups"], 0)
        post_rstd = pre_rstd = y = None
        if case["post"]:
            post_rstd = (b.square().sum(1) / width + EPS) ** -0.5
            b = b * post_rstd[:, None] * s["post_weight"].double()
        out = s["alpha"] * r + gate * b
        if case["pre"]:
            pre_rstd = (out.square().sum(1) / width + EPS) ** -0.5
            y = out * pre_rstd[:, None] * s["pre_weight"].double()
        return out, y, post_rstd, pre_rstd
    if op == "norm_backward":
        # through the Jacobian of x -> x rstd(x): rstd (I - u u^T / width), u = x rstd
        got = {}
        d = s["d_out"].double()
        if case["pre"]:
            k = s["pre_rstd"].double()[:, None]
            u, up = s["out"].double() * k, s["d_y"].double()
            got["d_pre_weight"] = torch.einsum("rc,rc->c", up, u)
            up = up * s["pre_weight"].double()
            d = d + k * (up - u * (torch.einsum("rc,rc->r", up, u) / width)[:, None])
        got["d_residual"] = s["alpha"] * d
        gate = s["gate"].double().repeat_interleave(rows // case["groups"], 0)
        if case["post"]:
            k = s["post_rstd"].double()[:, None]
            w = s["post_weight"].double()
            u = s["branch"].double() * k
            got["d_gate"] = (d * u * w).unflatten(0, (case["groups"], rows // case["groups"])).sum(1)
            up = d * gate
            got["d_post_weight"] = torch.einsum("rc,rc->c", up, u)
            up = up * w
            got["d_branch"] = k * (up - u * (torch.einsum("rc,rc->r", up, u) / width)[:, None])
        else:
            got["d_gate"] = (d * s["branch"].double()).unflatten(0, (case["groups"], rows // case["groups"])).sum(1)
            got["d_branch"] = d * gate
        return got
    if op == "quantize":
        # 2^ceil(log2(most / 448)), and the nearest e4m3 number (three bits below the leading one, steps of 2^-9 below 2^-6)
        x = s["x"].double()
        down, right = -rows % case["block_rows"], -width % BLOCK
        most = torch.nn.functional.pad(x.abs(), (0, right, 0, down)).unflatten(0, (-1, case["block_rows"])).unflatten(2, (-1, BLOCK)).amax((1, 3))
        # (a logarithm may fall on either side of a whole number, and a power next to its value: both are put right)
        power = lambda e: ((e.long() + 1023) << 52).view(torch.float64)  # noqa: E731
        e = torch.round(torch.log2(torch.where(most > 0, most, 1.0) / E4M3_MAX)).clamp(min=-126)
        e = torch.where(most > E4M3_MAX * power(e), e + 1, torch.where(most <= E4M3_MAX * power(e - 1), e - 1, e)).clamp(min=-126)
        scale = torch.where(most > 0, power(e), 1.0)
        v = x / scale.repeat_interleave(case["block_rows"], 0)[:rows].repeat_interleave(BLOCK, 1)[:, :width]
        _, e = torch.frexp(v.abs().clamp(min=2.0 ** -6))   # v = mantissa 2^e, mantissa in [1/2, 1)
        quantum = power(e - 4)
        return {"values": torch.round(v / quantum) * quantum, "scale": scale}   # (torch.round: ties to even)
    # the sum over blocks of 128 of (sum of products of the 8-bit numbers) times the two scales
    y = torch.zeros(rows, case["features"], dtype=torch.float64, device="cuda")
    row_block = torch.arange(case["features"], device="cuda") // BLOCK
    for k in range(-(-width // BLOCK)):
        part = s["xq"][:, k * BLOCK:(k + 1) * BLOCK].double() @ s["wq"][:, k * BLOCK:(k + 1) * BLOCK].double().t()
        y += part * s["x_scale"][:, k].double()[:, None] * s["w_scale"][row_block, k].double()
    return y
