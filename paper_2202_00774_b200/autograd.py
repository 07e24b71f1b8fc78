"""``torch.autograd`` front end: layers whose backward pass prunes the incoming output gradient
and computes the input gradient with the SDGP kernels (Algorithm 1; Section 3.1: "SDGP only
changes the data gradient; the weight gradient uses the unpruned dL/dO").

Only the data gradient runs in this library (and ReLU + 2 x 2 pooling, in one pass; and the operators of the language-model
layers at the end of this file). Convolutions,
matrix products and the weight gradient are the framework's own operators, which is the
integration the paper describes (Section 1: a drop-in change of the backward pass). Tensors are bf16 or fp16
CUDA tensors; convolutions use the channels-last memory format (its physical layout is the NHWC /
[Cout,R,S,Cin] layout of the C ABI, so nothing is copied or transposed).

Each of the first three layers comes in two forms with the same results. Plain calls (ordinary 16-bit CUDA tensors, integer arguments, nothing that
traces or transforms the call) run as C++ autograd functions (csrc/torch_autograd.cpp): a small layer's step is bound by
the host. Everything else runs as the Python autograd functions below: tensor subclasses and fake tensors, tracing and
compilation, function transforms, forward-mode differentiation, strides and paddings that are not one integer, other
devices and element types.

A step that is captured into a CUDA graph needs leaves without an eager graph that still lives: drop the outputs of earlier eager steps first.
torch keeps a leaf's gradient accumulator, with the stream that it was made on, for as long as any graph holds it, and waiting for that
stream inside a capture is an error that torch does not survive.
"""
from __future__ import annotations

import torch

from . import binding as _b

_CONV, _CONV_RELU, _CONV_RELU_POOL = 0, 1, 2


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return _b.BF16
    if t.dtype == torch.float16:
        return _b.FP16
    raise TypeError("SDGP layers take bfloat16 or float16 tensors, got %s" % t.dtype)


def _plain(x) -> bool:
    """Whether the C++ form may be asked (it makes the rest of the test and answers NotImplemented where it does not apply)."""
    return not torch.compiler.is_dynamo_compiling() and isinstance(x, torch.Tensor) and x.is_cuda


class _SDGPLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, n, m, scheme, seed):
        ctx.save_for_backward(x, weight)
        ctx.cfg = (n, m, scheme, seed)
        return x @ weight.t()

    @staticmethod
    def backward(ctx, grad_out):
        x, weight = ctx.saved_tensors
        n, m, scheme, seed = ctx.cfg
        dO = grad_out.reshape(-1, weight.shape[0]).contiguous()
        grad_x = grad_w = None
        if ctx.needs_input_grad[0]:
            rows, K = dO.shape
            N = weight.shape[1]
            dD = torch.empty((rows, N), dtype=dO.dtype, device=dO.device)
            ws = torch.empty(max(16, _b.sdgp_workspace_size_linear(rows, K, N)), dtype=torch.uint8, device=dO.device)
            # weight is [out_features, in_features] = [K, N]: the layout sdgp_dgrad_linear wants
            _b.sdgp_dgrad_linear_typed(dO, weight.contiguous(), dD, n, m, scheme, seed, _dtype_code(dO), workspace=ws)
            grad_x = dD.reshape(x.shape)
        if ctx.needs_input_grad[1]:
            grad_w = dO.t() @ x.reshape(-1, x.shape[-1])   # unpruned dL/dO (Section 3.1)
        return grad_x, grad_w, None, None, None, None


def sdgp_linear(x, weight, n=2, m=4, scheme=_b.MAGNITUDE, seed=0):
    """``x @ weight.T`` whose input gradient is ``prune(dL/dO) @ weight`` (N:M along out_features).
    in_features and out_features must be multiples of 64."""
    y = (_b._torch or _b._load()).linear_layer(x, weight, n, m, scheme, seed) if _plain(x) else NotImplemented
    return _SDGPLinearFn.apply(x, weight, n, m, scheme, seed) if y is NotImplemented else y


class _SDGPConv2dFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, stride, padding, n, m, scheme, seed):
        ctx.save_for_backward(x, weight)
        ctx.cfg = (stride, padding, n, m, scheme, seed)
        return torch.nn.functional.conv2d(x, weight, None, stride, padding)

    @staticmethod
    def backward(ctx, grad_out):
        x, weight = ctx.saved_tensors
        stride, padding, n, m, scheme, seed = ctx.cfg
        grad_x = grad_w = None
        if ctx.needs_input_grad[0]:
            # channels-last NCHW tensors are NHWC in memory: permuted views, no copies when the
            # tensors already have that format
            dO = grad_out.contiguous(memory_format=torch.channels_last).permute(0, 2, 3, 1)
            W = weight.contiguous(memory_format=torch.channels_last).permute(0, 2, 3, 1)   # [Cout,R,S,Cin]
            B, Cin, H, Wd = x.shape
            Cout, _, R, S = weight.shape
            dD = torch.empty((B, H, Wd, Cin), dtype=dO.dtype, device=dO.device)
            ws = torch.empty(max(16, _b.sdgp_workspace_size_conv2d(B, H, Wd, Cin, Cout, R, S, stride, padding)),
                             dtype=torch.uint8, device=dO.device)
            _b.sdgp_dgrad_conv2d_typed(dO, W, dD, stride, padding, n, m, scheme, seed, _dtype_code(dO), workspace=ws)
            grad_x = dD.permute(0, 3, 1, 2)   # NCHW view of channels-last storage
        if ctx.needs_input_grad[1]:
            grad_w = torch.nn.grad.conv2d_weight(x, weight.shape, grad_out, stride, padding)   # unpruned dL/dO
        return grad_x, grad_w, None, None, None, None, None, None


def sdgp_conv2d(x, weight, stride=1, padding=0, n=2, m=4, scheme=_b.MAGNITUDE, seed=0):
    """``conv2d(x, weight)`` (NCHW tensors, channels-last storage recommended, no bias, stride 1 or 2,
    one padding value for both axes) whose input gradient is computed from dL/dO pruned N:M along
    the output channels. Channel counts must be multiples of 64."""
    y = (_b._torch or _b._load()).conv2d_layer(x, weight, stride, padding, _CONV, n, m, scheme, seed) if _plain(x) else NotImplemented
    return _SDGPConv2dFn.apply(x, weight, stride, padding, n, m, scheme, seed) if y is NotImplemented else y


class _SDGPConv2dReLUFn(torch.autograd.Function):
    """``relu(conv2d(x, weight))``, optionally followed by 2 x 2 max pooling. The backward pass forms the
    convolution's dL/dO from the gradient above the ReLU (or above the pooling) with the library's producer, which
    writes the unpruned dL/dO - the weight gradient's operand (Section 3.1) - and its compressed pruned copy in one
    pass; the sparse contraction then gives the input gradient (Section 2.1, Fig. 2)."""

    @staticmethod
    def forward(ctx, x, weight, stride, padding, pool, n, m, scheme, seed):
        act = torch.relu(torch.nn.functional.conv2d(x, weight, None, stride, padding))
        act = act.contiguous(memory_format=torch.channels_last)
        ctx.save_for_backward(x, weight, act)
        ctx.cfg = (stride, padding, pool, n, m, scheme, seed)
        return torch.nn.functional.max_pool2d(act, 2) if pool else act

    @staticmethod
    def backward(ctx, grad_out):
        x, weight, act = ctx.saved_tensors
        stride, padding, pool, n, m, scheme, seed = ctx.cfg
        dt = _dtype_code(grad_out)
        B, Cin, H, Wd = x.shape
        Cout, _, R, S = weight.shape
        P, Q = act.shape[2], act.shape[3]
        dY = grad_out.contiguous(memory_format=torch.channels_last).permute(0, 2, 3, 1)   # NHWC views
        a = act.permute(0, 2, 3, 1)
        dO = torch.empty((B, P, Q, Cout), dtype=dY.dtype, device=dY.device)
        compressed = n <= 2 and Cout % 128 == 0 and ctx.needs_input_grad[0]
        vals = torch.empty((B, P, Q, Cout // 2), dtype=dY.dtype, device=dY.device) if compressed else None
        meta = torch.empty((B, P, Q, Cout // 16), dtype=torch.int16, device=dY.device) if compressed else None
        pn, pm = (n, m) if compressed else (4, 4)   # n == m: nothing is pruned, the producer only writes dL/dO
        if pool:
            _b.sdgp_maxpool_relu_backward_prune(dY, a, pn, pm, scheme, seed, dt, grad=dO, values=vals, meta=meta)
        else:
            _b.sdgp_relu_backward_prune(dY, a, pn, pm, scheme, seed, dt, grad=dO, values=vals, meta=meta)
        grad_x = grad_w = None
        if ctx.needs_input_grad[0]:
            W = weight.contiguous(memory_format=torch.channels_last).permute(0, 2, 3, 1)   # [Cout,R,S,Cin]
            dD = torch.empty((B, H, Wd, Cin), dtype=dY.dtype, device=dY.device)
            if compressed:
                _b.sdgp_spmm_conv2d_typed(vals, meta, W, dD, stride, padding, dt)
            else:   # no compressed form to hand over: prune dL/dO in a pass of its own
                ws = torch.empty(max(16, _b.sdgp_workspace_size_conv2d(B, H, Wd, Cin, Cout, R, S, stride, padding,
                                                                       _b.FLAG_TWO_PASS if n <= 2 else _b.FLAG_MASKED)),
                                 dtype=torch.uint8, device=dY.device)
                _b.sdgp_dgrad_conv2d_typed(dO, W, dD, stride, padding, n, m, scheme, seed, dt, workspace=ws,
                                           flags=_b.FLAG_TWO_PASS if n <= 2 else _b.FLAG_MASKED)
            grad_x = dD.permute(0, 3, 1, 2)
        if ctx.needs_input_grad[1]:
            grad_w = torch.nn.grad.conv2d_weight(x, weight.shape, dO.permute(0, 3, 1, 2), stride, padding)   # unpruned dL/dO
        return grad_x, grad_w, None, None, None, None, None, None, None


def sdgp_conv2d_relu(x, weight, stride=1, padding=0, pool=False, n=2, m=4, scheme=_b.MAGNITUDE, seed=0):
    """``relu(conv2d(x, weight))`` - with ``pool=True`` followed by ``max_pool2d(., 2)`` - whose backward pass
    forms and prunes the convolution's dL/dO in one pass over the incoming gradient (ReLU backward, pooling
    backward and Algorithm 1 together), computes the input gradient from the pruned copy and the weight gradient
    from the unpruned one (Section 3.1). Same tensor requirements as ``sdgp_conv2d``; with ``pool=True`` the
    convolution's output height and width must be even."""
    y = NotImplemented
    if _plain(x):
        y = (_b._torch or _b._load()).conv2d_layer(x, weight, stride, padding, _CONV_RELU_POOL if pool else _CONV_RELU, n, m, scheme, seed)
    return _SDGPConv2dReLUFn.apply(x, weight, stride, padding, pool, n, m, scheme, seed) if y is NotImplemented else y


# ---- a language model's layers around the pruned data gradient (Python forms only: their steps are not bound by the host) ----


def _linear_grads(ctx, dO, vals, meta, x, weight, need_x, need_w, pattern):
    """Input and weight gradient of ``x @ weight.T`` from the unpruned dL/dO [rows, K] and, where the pass that made it has
    written one, its compressed pruned copy. Both products are of dL/dO's type: weights or activations of another one (fp32 weights of
    the 8-bit layer, operands that autocast has rounded) are rounded to it."""
    n, m, scheme, seed = pattern
    grad_x = grad_w = None
    if need_x:
        rows, K = dO.shape
        N = weight.shape[1]
        dt = _dtype_code(dO)
        W = weight.to(dO.dtype).contiguous()
        dD = torch.empty((rows, N), dtype=dO.dtype, device=dO.device)
        with torch.cuda.device(dO.device):
            if vals is not None:
                _b.sdgp_spmm_linear_typed(vals, meta, W, dD, dt)
            else:
                flags = _b.FLAG_TWO_PASS if n <= 2 or n == m else _b.FLAG_MASKED
                ws = torch.empty(max(16, _b.sdgp_workspace_size_linear(rows, K, N, flags)), dtype=torch.uint8, device=dO.device)
                _b.sdgp_dgrad_linear_typed(dO, W, dD, n, m, scheme, seed, dt, workspace=ws, flags=flags)
        grad_x = dD.reshape(x.shape).to(x.dtype)
    if need_w:
        grad_w = (dO.t() @ x.reshape(-1, x.shape[-1]).to(dO.dtype)).to(weight.dtype)   # unpruned dL/dO (Section 3.1)
    return grad_x, grad_w


def _compressed(rows, K, n, need_x, like):
    """Outputs for the compressed pruned copy of dL/dO [rows, K], where the sparse contraction can take it."""
    if n > 2 or K % 128 != 0 or not need_x:
        return None, None
    return (torch.empty((rows, K // 2), dtype=like.dtype, device=like.device),
            torch.empty((rows, K // 16), dtype=torch.int16, device=like.device))


class _SDGPLinearLogprobFn(torch.autograd.Function):
    """The head of a language model: ``x @ weight.T`` and the log probabilities of the targets. The backward pass forms the
    logits' gradient - the first dL/dO of the backward chain - and its compressed pruned copy in one pass."""

    @staticmethod
    def forward(ctx, x, weight, targets, classes, n, m, scheme, seed):
        ctx.set_materialize_grads(False)
        logits = (x @ weight.t()).reshape(-1, weight.shape[0])
        t = targets.reshape(-1).contiguous()
        rows = logits.shape[0]
        logprob, entropy, lse = (torch.empty(rows, dtype=torch.float32, device=x.device) for _ in range(3))
        _b.sdgp_token_logprob(logits, t, logprob, entropy=entropy, lse=lse, classes=classes, dtype=_dtype_code(logits))
        ctx.save_for_backward(x, weight, logits, t, lse, entropy)
        ctx.cfg = (classes, n, m, scheme, seed)
        return logprob.reshape(targets.shape), entropy.reshape(targets.shape)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_logprob, d_entropy):
        x, weight, logits, t, lse, entropy = ctx.saved_tensors
        classes, n, m, scheme, seed = ctx.cfg
        if d_logprob is None and d_entropy is None:
            return (None,) * 8
        need_x, need_w = ctx.needs_input_grad[:2]
        flat = lambda g: None if g is None else g.reshape(-1).float().contiguous()  # noqa: E731
        rows, K = logits.shape
        dO = torch.empty_like(logits)
        vals, meta = _compressed(rows, K, n, need_x, logits)
        _b.sdgp_token_logprob_backward(logits, t, lse, flat(d_logprob), grad=dO, entropy=entropy, d_entropy=flat(d_entropy), n=n, m=m,
                                       scheme=scheme, seed=seed, dtype=_dtype_code(logits), values=vals, meta=meta, classes=classes)
        return (*_linear_grads(ctx, dO, vals, meta, x, weight, need_x, need_w, (n, m, scheme, seed)), None, None, None, None, None, None)


def sdgp_linear_logprob(x, weight, targets, classes=None, n=2, m=4, scheme=_b.MAGNITUDE, seed=0):
    """Log probabilities of ``targets`` (int64, the shape of ``x`` without its last dimension; negative: not counted, 0) under the
    logits ``x @ weight.T``, and the entropy of every position: two float32 tensors of the shape of ``targets``. ``weight`` has one
    row for each token; rows past ``classes`` (default: none) are padding to a multiple of 64 and get no probability. The logits'
    gradient is formed and pruned N:M along the tokens (in one pass, where n <= 2 and ``weight`` has a multiple of 128 rows); ``x``'s gradient
    is computed from the pruned copy, the weights' from the unpruned one. Where ``x`` takes a gradient, in_features and the rows of ``weight``
    must be multiples of 64 and m 4, 8, 16 or 32: the backward pass refuses others, as ``sdgp_linear``'s does."""
    return _SDGPLinearLogprobFn.apply(x, weight, targets, weight.shape[0] if classes is None else classes, n, m, scheme, seed)


class _SDGPLinearResidualNormFn(torch.autograd.Function):
    """The last layer of a block and the boundary to the next one. The backward pass writes the layer's dL/dO and its
    compressed pruned copy in the pass that goes back through norms, gate and residual sum."""

    @staticmethod
    def forward(ctx, x, weight, residual, post_weight, pre_weight, gate, alpha, eps, n, m, scheme, seed):
        ctx.set_materialize_grads(False)
        branch = (x @ weight.t()).reshape(-1, weight.shape[0])
        r = residual.reshape(branch.shape).contiguous()
        c = lambda w: None if w is None else w.contiguous()  # noqa: E731
        wp, wn, g = c(post_weight), c(pre_weight), c(gate)
        f32 = dict(dtype=torch.float32, device=x.device)
        post_rstd = torch.empty(branch.shape[0], **f32) if wp is not None else None
        pre_rstd = torch.empty(branch.shape[0], **f32) if wn is not None else None
        out = torch.empty_like(branch)
        y = torch.empty_like(branch) if wn is not None else None
        _b.sdgp_residual_norm(branch, r, out, y, post_weight=wp, gate=g, pre_weight=wn, alpha=alpha, eps=eps, dtype=_dtype_code(branch),
                              post_rstd=post_rstd, pre_rstd=pre_rstd)
        out = out.reshape(residual.shape)
        y = None if y is None else y.reshape(residual.shape)
        ctx.save_for_backward(x, weight, wp, wn, g, branch, out, post_rstd, pre_rstd)
        ctx.cfg = (alpha, n, m, scheme, seed)
        return out, y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_out, d_y):
        x, weight, wp, wn, g, branch, out, post_rstd, pre_rstd = ctx.saved_tensors
        alpha, n, m, scheme, seed = ctx.cfg
        if d_out is None and d_y is None:
            return (None,) * 12
        need = ctx.needs_input_grad
        flat = lambda t: None if t is None else t.reshape(branch.shape).contiguous()  # noqa: E731
        rows, C = branch.shape
        f32 = dict(dtype=torch.float32, device=x.device)
        d_branch = torch.empty_like(branch) if need[0] or need[1] else None
        d_residual = torch.empty_like(branch) if need[2] else None
        d_post = torch.empty(C, **f32) if need[3] and wp is not None else None
        d_pre = torch.zeros(C, **f32) if need[4] and wn is not None else None
        d_gate = torch.empty(g.shape, **f32) if need[5] and g is not None else None
        vals, meta = _compressed(rows, C, n, need[0], branch)
        groups = 1 if g is None else g.numel() // C
        ws = torch.empty(max(16, _b.sdgp_workspace_size_residual_norm_backward(rows, C, groups)), dtype=torch.uint8, device=x.device)
        _b.sdgp_residual_norm_backward(branch, out.reshape(branch.shape), flat(d_out), flat(d_y), post_weight=wp, gate=g,
                                       pre_weight=wn if d_y is not None else None, post_rstd=post_rstd,
                                       pre_rstd=pre_rstd if d_y is not None else None, alpha=alpha, n=n, m=m, scheme=scheme, seed=seed,
                                       dtype=_dtype_code(branch), d_residual=d_residual, d_branch=d_branch, d_gate=d_gate,
                                       d_post_weight=d_post, d_pre_weight=d_pre if d_y is not None else None, values=vals, meta=meta,
                                       workspace=ws)
        like = lambda t, w: None if t is None else t.to(w.dtype).reshape(w.shape)  # noqa: E731
        grad_x, grad_w = _linear_grads(ctx, d_branch, vals, meta, x, weight, need[0], need[1], (n, m, scheme, seed))
        return (grad_x, grad_w, None if d_residual is None else d_residual.reshape(out.shape), like(d_post, wp), like(d_pre, wn),
                like(d_gate, g), None, None, None, None, None, None)


def sdgp_linear_residual_norm(x, weight, residual, post_weight=None, pre_weight=None, gate=None, alpha=1.0, eps=1e-6, n=2, m=4,
                              scheme=_b.MAGNITUDE, seed=0):
    """The last linear layer of a block with the boundary to the next block:
    ``out = alpha * residual + gate * norm(x @ weight.T) * post_weight`` and ``y = norm(out) * pre_weight`` (root mean square norms;
    without ``post_weight`` the branch is not normalised, without ``pre_weight`` ``y`` is None). ``gate`` has one row, one for each
    of equal runs of positions (sequences), or one for every position: its rows are taken in order, whatever its leading dimensions, and not
    broadcast. ``residual``, the norms' weights and ``gate`` are of the product's element type (bf16 or fp16); others, float32 among them,
    are refused. Returns ``(out, y)``. The layer's dL/dO is formed and pruned N:M along its output features (in one pass, where n <= 2 and
    out_features is a multiple of 128); gradients of weights and gate are summed in float32. Where ``x`` takes a gradient, in_features and
    out_features must be multiples of 64 and m 4, 8, 16 or 32: the backward pass refuses others, as ``sdgp_linear``'s does."""
    return _SDGPLinearResidualNormFn.apply(x, weight, residual, post_weight, pre_weight, gate, alpha, eps, n, m, scheme, seed)


def sdgp_fp8_weights(weight):
    """``weight`` [out_features, in_features] in e4m3 with a scale for each 128 x 128 block, as ``sdgp_linear_fp8`` takes it: for
    steps that use the same weights more than once."""
    w = weight.detach().contiguous()
    q = torch.empty(w.shape, dtype=torch.float8_e4m3fn, device=w.device)
    scale = torch.empty((-(-w.shape[0] // 128), -(-w.shape[1] // 128)), dtype=torch.float32, device=w.device)
    _b.sdgp_fp8_quantize(w, q, scale, block_rows=128, dtype=_b.FP32 if w.dtype == torch.float32 else _dtype_code(w))
    return q, scale


class _SDGPLinearFp8Fn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, wq, w_scale, n, m, scheme, seed):
        ctx.save_for_backward(x, weight)
        ctx.cfg = (n, m, scheme, seed)
        rows_of_x = x.reshape(-1, x.shape[-1]).contiguous()
        rows, K = rows_of_x.shape
        xq = torch.empty((rows, K), dtype=torch.float8_e4m3fn, device=x.device)
        x_scale = torch.empty((rows, -(-K // 128)), dtype=torch.float32, device=x.device)
        _b.sdgp_fp8_quantize(rows_of_x, xq, x_scale, dtype=_dtype_code(x))
        y = torch.empty((rows, wq.shape[0]), dtype=x.dtype, device=x.device)
        _b.sdgp_fp8_linear(xq, x_scale, wq, w_scale, y, dtype=_dtype_code(x))
        return y.reshape(*x.shape[:-1], wq.shape[0])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out):
        x, weight = ctx.saved_tensors
        dO = grad_out.reshape(-1, weight.shape[0]).contiguous()
        return (*_linear_grads(ctx, dO, None, None, x, weight, *ctx.needs_input_grad[:2], ctx.cfg), None, None, None, None, None, None)


def sdgp_linear_fp8(x, weight, quantized=None, n=2, m=4, scheme=_b.MAGNITUDE, seed=0):
    """``x @ weight.T`` in 8 bits - both quantised to e4m3 with a scale for each block of 128 - whose backward pass is that of
    ``sdgp_linear``: the roundings pass the gradient through, the input gradient is ``prune(dL/dO) @ weight`` in 16 bits, the
    weight gradient uses the unpruned dL/dO. ``quantized``: what ``sdgp_fp8_weights(weight)`` gave. in_features and out_features
    must be multiples of 64. ``x`` is bf16 or fp16; ``weight`` may be of another type (fp32 master weights): it is quantised as it is, and
    rounded to ``x``'s type for the input gradient."""
    wq, w_scale = sdgp_fp8_weights(weight) if quantized is None else quantized
    if wq.shape != weight.shape:
        raise ValueError(f"sdgp_linear_fp8: quantized weights of shape {tuple(wq.shape)} for weights of shape {tuple(weight.shape)}")
    return _SDGPLinearFp8Fn.apply(x, weight, wq, w_scale, n, m, scheme, seed)
