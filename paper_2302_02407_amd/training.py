"""A training step around the distillation loss, in the clear (sequencing and buffers only).

What a student of polynomial activations, or its teacher, is trained with beside `distill.distill_loss`, each differentiable:

    y, h = layer_norm(ctx, x, weight, bias, residual=r)      # h = x + r goes on along the residual path
    u = linear_q8(ctx, y, w)                                 # keeps y in 8 bits for w's gradient
    a = polynomial(ctx, u, coefs)                            # sum of coefs[i] u^i, keeps u in 8 bits
    logp, entropy, values, index = token_logprobs(ctx, z, tokens, k=8)

What is kept in 8 bits takes 1.01 bytes an element between the forward and the backward pass, and the gradients that need it are those at the
values that are kept: off by at most 2^-4 of themselves, or 2^-10 of the power of two that 128 columns share.

Rows are the last dimension's.  `ctx` is an HEContext; its calls go to the stream that was current at its creation, so these functions want that stream to be
the current one, in the backward pass too.
"""
import torch
import torch.nn.functional as F

from .distill import _code_rows, _same_stream

BLOCK = 128


def _own_rows(x):
    """x as a matrix whose rows are in one piece and share nothing."""
    m = x.reshape(-1, x.shape[-1])
    if m.numel() == 0:
        return m.clone(memory_format=torch.contiguous_format)    # nothing may have any strides
    return m if (m.stride(1) == 1 or m.shape[1] == 1) and (m.shape[0] <= 1 or m.stride(0) >= m.shape[1]) else m.contiguous()


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(run, x, residual, weight, bias, ctx, eps):
        _same_stream(ctx)
        run.set_materialize_grads(False)
        h = torch.empty(x.shape, dtype=x.dtype, device=x.device) if residual is not None else x
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        stats = torch.empty((x.shape[0], 4), dtype=torch.float32, device=x.device)
        ctx.he_layernorm(x, y, eps, weight=weight, bias=bias, residual=residual, sum_out=h if residual is not None else None, stats=stats)
        run.save_for_backward(h, stats, weight, bias)
        run.ctx, run.residual = ctx, residual is not None
        return (y, h) if residual is not None else y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(run, dy, dsum=None):
        h, stats, weight, bias = run.saved_tensors
        _same_stream(run.ctx)
        if dy is None:                                        # only the sum has a gradient
            if dsum is None:
                return (None,) * 6
            none = [torch.zeros_like(p) if p is not None and n else None for p, n in zip((weight, bias), run.needs_input_grad[2:4])]
            return dsum, dsum, *none, None, None
        dx = torch.empty(h.shape, dtype=h.dtype, device=h.device)
        dweight, dbias = (torch.empty_like(p) if p is not None and n else None for p, n in zip((weight, bias), run.needs_input_grad[2:4]))
        run.ctx.he_layernorm_grad(h, stats, _own_rows(dy), dx, weight=weight, dsum=None if dsum is None else _own_rows(dsum), dweight=dweight, dbias=dbias)
        return dx, dx if run.residual else None, dweight, dbias, None, None


def layer_norm(ctx, x, weight=None, bias=None, eps=1e-5, residual=None):
    """The layer norm of x's rows; with a residual that of x + residual, and that sum too."""
    rows = _own_rows(x)
    more = _own_rows(residual.expand_as(x)) if residual is not None else None
    out = _LayerNorm.apply(rows, more, weight, bias, ctx, eps)
    return tuple(t.view(x.shape) for t in out) if residual is not None else out.view(x.shape)


def keep_q8(ctx, x, coefs=None, y=None):
    """Codes and the bytes of their powers of rows x, and with coefficients the polynomial in y."""
    codes = _code_rows(*x.shape, x.device)
    exponents = torch.empty((x.shape[0], -(-x.shape[1] // BLOCK)), dtype=torch.uint8, device=x.device)
    ctx.he_poly_q8(x, codes, exponents, coefs=coefs, y=y)
    return codes, exponents


class _Polynomial(torch.autograd.Function):
    @staticmethod
    def forward(run, u, coefs, ctx):
        _same_stream(ctx)
        y = torch.empty(u.shape, dtype=u.dtype, device=u.device)
        codes, exponents = keep_q8(ctx, u, coefs, y)
        run.save_for_backward(codes, exponents, coefs)
        run.ctx = ctx
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(run, dy):
        codes, exponents, coefs = run.saved_tensors
        _same_stream(run.ctx)
        du = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
        dcoefs = torch.empty_like(coefs) if run.needs_input_grad[1] else None
        run.ctx.he_poly_grad_q8(codes, exponents, coefs, _own_rows(dy), du, dcoefs=dcoefs)
        return du, dcoefs, None


def polynomial(ctx, u, coefs):
    """sum of coefs[i] u^i, up to 9 coefficients of 32 bits; u is kept in 8 bits for the backward pass."""
    return _Polynomial.apply(_own_rows(u), coefs.contiguous(), ctx).view(u.shape)


class _LinearQ8(torch.autograd.Function):
    @staticmethod
    def forward(run, x, weight, ctx, mixed):
        _same_stream(ctx)
        run.ctx, run.kept = ctx, run.needs_input_grad[1]
        run.save_for_backward(weight, *(keep_q8(ctx, x) if run.kept else ()))
        return F.linear(x, weight.to(x.dtype) if mixed else weight)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(run, dy):
        weight, *kept = run.saved_tensors
        _same_stream(run.ctx)
        dy, dweight = _own_rows(dy), None
        if run.kept:
            dweight = torch.empty(weight.shape, dtype=weight.dtype, device=weight.device)
            run.ctx.he_weight_grad_q8(dy, *kept, dweight)
        with torch.autocast("cuda", enabled=False):           # the forward pass says in which type
            return dy @ weight.to(dy.dtype) if run.needs_input_grad[0] else None, dweight, None, None


def linear_q8(ctx, x, weight):
    """x times weight [n][k <= 65536] transposed, by the library's product; x is kept in 8 bits for the weight's gradient.  Under autocast x and the product are of its type, and the weight's
    gradient, of the weight's own, is not rounded to that."""
    rows, mixed = _own_rows(x), torch.is_autocast_enabled("cuda") and x.dtype != torch.float64
    if mixed:                                                 # here and not by autocast, which would keep the weight's copy, made without a gradient, for others in its region
        rows = rows.to(torch.get_autocast_dtype("cuda"))
    return _LinearQ8.apply(rows, weight, ctx, mixed).view(*x.shape[:-1], weight.shape[0])


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(run, z, ctx, tokens, tau, k):
        _same_stream(ctx)
        run.set_materialize_grads(False)
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=z.device)  # noqa: E731
        rows = z.shape[0]
        logp, entropy, stats = new(rows), new(rows), new(rows, 4) if run.needs_input_grad[0] else None
        values, index = (new(rows, k), new(rows, k, dtype=torch.int32)) if k else (None, None)
        ctx.he_token_logprobs(z, tau, tokens=tokens, logp=logp, entropy=entropy, values=values, index=index, stats=stats)
        run.save_for_backward(z, stats, tokens)
        run.ctx, run.tau = ctx, tau
        if k:
            run.mark_non_differentiable(values, index)
        return logp, entropy, values, index

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(run, dlogp, dentropy, dvalues, dindex):
        z, stats, tokens = run.saved_tensors
        _same_stream(run.ctx)
        grad = torch.empty(z.shape, dtype=z.dtype, device=z.device)
        of = lambda g: None if g is None else g.contiguous()  # noqa: E731
        run.ctx.he_token_logprobs_grad(z, run.tau, stats, grad, tokens=tokens, logp_weights=of(dlogp), entropy_weights=of(dentropy))
        return grad, None, None, None, None


def token_logprobs(ctx, z, tokens, tau=1.0, k=0):
    """Of softmax(z / tau), row by row: the log probability of a token (int32, or int64; one outside the vocabulary, as -1 for padding, has 0 and no gradient) and the
    entropy, both differentiable; log probability and index of the k most probable ones (None without k), which are not."""
    if tokens.dtype == torch.int64:
        tokens = tokens.clamp(-1, z.shape[-1]).to(torch.int32)
    shape = z.shape[:-1]
    logp, entropy, values, index = _TokenLogprobs.apply(_own_rows(z), ctx, tokens.reshape(-1).contiguous(), tau, k)
    return logp.view(shape), entropy.view(shape), *(None if t is None else t.view(*shape, k) for t in (values, index))
