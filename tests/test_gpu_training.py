"""A training step from the operators as they are used: differentiable functions, layer by layer against 64 bits, in a captured graph and on odd tensors."""
import math

import pytest
import torch

import plain_ref as R
import train_ref as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    return HEContext.from_params(config_params(0))


def near(got, want, size, dtype, by=2.0 ** -15):
    off = (got.detach().cpu().double().reshape(want.shape) - want).abs()
    bound = by * size + T.rounding(want, dtype)
    assert (off <= bound).all(), float((off / bound).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_step_layer_by_layer(ctx, dtype):
    """Norm with a residual, a layer, the polynomial, a second layer beside the residual path, log probabilities.  Every layer's gradients against their definitions from the
    layer's own input and the gradient that reached its output."""
    from paper_2302_02407_amd.training import layer_norm, linear_q8, polynomial, token_logprobs
    g, batch, length, dim, hidden, vocab = T.rng(1), 3, 17, 200, 130, 500
    new = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    leaves = {"x": new(batch, length, dim).to(dtype), "r": new(batch, length, dim).to(dtype), "nw": 1 + 0.1 * new(dim), "nb": 0.1 * new(dim),
              "w1": (new(hidden, dim) / dim ** 0.5).to(dtype), "c": torch.tensor([0.1, 0.9, 0.3, -0.1]), "w2": (new(vocab, hidden) / hidden ** 0.5).to(dtype)}
    p = {n: t.cuda().requires_grad_() for n, t in leaves.items()}
    tokens = torch.randint(-1, vocab, (batch, length), generator=g)
    wl, wh, wr = new(batch, length), 0.1 * new(batch, length), new(batch, length, dim).to(dtype)
    y, h = layer_norm(ctx, p["x"], p["nw"], p["nb"], residual=p["r"])
    u = linear_q8(ctx, y, p["w1"])
    a = polynomial(ctx, u, p["c"])
    z = linear_q8(ctx, a, p["w2"])
    logp, entropy, values, index = token_logprobs(ctx, z, tokens.cuda(), 1.3, k=5)
    loss = (logp * wl.cuda()).sum() + (entropy * wh.cuda()).sum() + (h * wr.cuda()).sum()
    for t in (y, h, u, a, z):
        t.retain_grad()
    loss.backward()
    flat = lambda t: t.detach().cpu().reshape(-1, t.shape[-1])  # noqa: E731

    lp, _, ent = T.distribution(flat(z), 1.3)
    there = tokens.reshape(-1) >= 0
    want = torch.where(there, lp.gather(1, tokens.reshape(-1).clamp_min(0)[:, None])[:, 0], 0.0)
    assert ((logp.detach().cpu().double().reshape(-1) - want).abs() <= 1e-5 + 2.0 ** -22 * want.abs()).all()
    assert torch.equal(index.cpu().reshape(-1, 5).long(), T.top_order(flat(z), 5)) and not values.requires_grad
    dz, size = T.logprobs_grad(flat(z), 1.3, tokens.reshape(-1), wl.reshape(-1), wh.reshape(-1))
    near(z.grad, dz, size, dtype, 2e-5)

    def layer(x, weight, out):
        """What is kept of x, exactly; a library product of k terms in 32 bits."""
        kept, d = T.kept(*T.keep(flat(x).float())), flat(out.grad).double()
        near(p[weight].grad, d.T @ kept, d.abs().T @ kept.abs(), dtype, (len(d) + 16) * 2.0 ** -24)
        w = leaves[weight].double()
        near(x.grad, d @ w, d.abs() @ w.abs(), dtype, (w.shape[0] + 16) * 2.0 ** -24)

    layer(a, "w2", z)
    du, dc, size, size_c = T.poly_grad(T.kept(*T.keep(flat(u).float())), leaves["c"], flat(a.grad))
    near(u.grad, du, size, dtype, 2.0 ** -19)
    near(p["c"].grad, dc, size_c, torch.float32, 2.0 ** -19)
    layer(y, "w1", u)
    assert torch.equal(flat(h), (flat(leaves["x"]).float() + flat(leaves["r"]).float()).to(dtype)) and torch.equal(flat(h.grad), flat(wr))
    dx, dw, db, size, size_w, size_b = T.norm_grad(flat(h), flat(y.grad), leaves["nw"], flat(wr), 1e-5)
    near(p["x"].grad, dx, size, dtype)
    assert torch.equal(p["x"].grad, p["r"].grad)
    near(p["nw"].grad, dw, size_w, torch.float32)
    near(p["nb"].grad, db, size_b, torch.float32)


def test_inputs_that_share_or_skip_memory(ctx):
    """Every second column, a row for all, a transposed matrix, gradients of one number for all: as contiguous ones."""
    from paper_2302_02407_amd.training import layer_norm, linear_q8, polynomial, token_logprobs
    g = T.rng(2)
    base, weight, c = torch.randn((12, 80), generator=g).cuda(), torch.randn((7, 40), generator=g).cuda(), torch.tensor([0.0, 1.0, 0.5], device="cuda")
    tokens = torch.arange(12, device="cuda") % 40
    calls = [lambda t: layer_norm(ctx, t), lambda t: layer_norm(ctx, t, residual=t[:1])[0], lambda t: polynomial(ctx, t, c), lambda t: linear_q8(ctx, t, weight),
             lambda t: token_logprobs(ctx, t, tokens)[0], lambda t: token_logprobs(ctx, t, tokens)[1]]
    for view in (lambda t: t[:, ::2], lambda t: t[:1, :40].expand(12, 40), lambda t: t.view(-1)[:480].view(40, 12).t(), lambda t: t[:, 3:43]):
        for call in calls:
            one, two = base.clone().requires_grad_(), base.clone().requires_grad_()
            a, b = call(view(one)), call(view(two).contiguous())
            assert torch.equal(a, b)
            a.sum().backward()                                # a gradient of stride 0
            (b * torch.ones_like(b)).sum().backward()
            assert torch.equal(one.grad, two.grad)


def test_what_is_not_asked_for(ctx):
    """Gradients by parameters alone, by the input alone, by the sum alone; no rows."""
    from paper_2302_02407_amd.training import layer_norm, linear_q8, polynomial, token_logprobs
    g = T.rng(3)
    x, r = torch.randn((9, 64), generator=g).cuda(), torch.randn((9, 64), generator=g).cuda()
    w = torch.ones(64, device="cuda", requires_grad=True)
    layer_norm(ctx, x, w).sum().backward()
    assert w.grad is not None and x.grad is None
    w.grad, leaf = None, x.clone().requires_grad_()
    y, h = layer_norm(ctx, leaf, w, residual=r)
    h.sum().backward()
    assert (leaf.grad == 1).all() and (w.grad == 0).all()
    weight = torch.randn((5, 64), generator=g).cuda().requires_grad_()
    linear_q8(ctx, x, weight).sum().backward()
    near(weight.grad, T.kept(*T.keep(x.cpu())).sum(dim=0).expand(5, 64), x.cpu().double().abs().sum(dim=0).expand(5, 64), torch.float32, 25 * 2.0 ** -24)
    linear_q8(ctx, leaf, weight.detach()).sum().backward()
    z = torch.randn((4, 30), generator=g).cuda().requires_grad_()
    logp, entropy, values, index = token_logprobs(ctx, z, torch.tensor([3, -1, 30, 2 ** 40], device="cuda"))
    assert values is None and index is None and (logp[1:] == 0).all()
    logp.sum().backward()
    assert (z.grad[1:] == 0).all() and (z.grad[0] != 0).any()
    e = torch.zeros((0, 64), device="cuda", requires_grad=True)
    (layer_norm(ctx, e, w).sum() + polynomial(ctx, e, torch.ones(2, device="cuda")).sum() + linear_q8(ctx, e, weight).sum()).backward()
    assert e.grad.shape == (0, 64)


@pytest.mark.parametrize("low", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("inside", [True, False])
def test_layer_in_mixed_precision(ctx, low, inside):
    """Parameters of 32 bits under autocast: the product in 16 bits, the weight's gradient in 32, whether the backward pass runs in the region or behind it; a second use of the weight there
    by torch's own product has its gradient too."""
    from paper_2302_02407_amd.training import linear_q8
    g, m, n, k = T.rng(6), 37, 50, 200
    x, w, wr = torch.randn((m, k), generator=g), torch.randn((n, k), generator=g) / 16, torch.randn((m, n), generator=g)
    px, pw = x.cuda().requires_grad_(), w.cuda().requires_grad_()
    with torch.autocast("cuda", dtype=low):
        u = linear_q8(ctx, px, pw)
        assert u.dtype == low
        if inside:
            u.backward(wr.to(low).cuda())
    if not inside:
        u.backward(wr.to(low).cuda())
    assert px.grad.dtype == pw.grad.dtype == torch.float32
    a, b, d = x.to(low).double(), w.to(low).double(), wr.to(low).double()
    near(u, a @ b.T, a.abs() @ b.abs().T, low, (k + 16) * 2.0 ** -24)
    near(px.grad, d @ b, d.abs() @ b.abs(), low, (n + 16) * 2.0 ** -24)
    kept = T.kept(*T.keep(x.to(low).float()))
    near(pw.grad, d.T @ kept, d.abs().T @ kept.abs(), torch.float32, (m + 16) * 2.0 ** -24)
    pw.grad = None
    with torch.autocast("cuda", dtype=low):
        linear_q8(ctx, px, pw.detach()).sum().backward()
        u = linear_q8(ctx, px, pw)
        (u.sum() + torch.nn.functional.linear(px, pw).sum()).backward()
    one = pw.grad.clone()
    pw.grad = None
    with torch.autocast("cuda", dtype=low):
        linear_q8(ctx, px, pw).sum().backward()
    layer = pw.grad.clone()
    near(one - layer, a.sum(dim=0).expand(n, k), a.abs().sum(dim=0).expand(n, k) + layer.cpu().double().abs(), low, (m + 16) * 2.0 ** -24)


def test_layer_behind_a_region_of_mixed_precision(ctx):
    """A forward pass of 32 bits has a backward pass of 32 bits, also where that runs under autocast."""
    from paper_2302_02407_amd.training import linear_q8
    g = T.rng(7)
    x, w, d = torch.randn((20, 64), generator=g).cuda().requires_grad_(), torch.randn((30, 64), generator=g).cuda(), torch.randn((20, 30), generator=g).cuda()
    u = linear_q8(ctx, x, w)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        u.backward(d)
    a, b = d.cpu().double(), w.cpu().double()
    near(x.grad, a @ b, a.abs() @ b.abs(), torch.float32, 46 * 2.0 ** -24)


def test_another_stream_is_refused(ctx):
    from paper_2302_02407_amd.training import layer_norm
    x = torch.zeros((4, 64), device="cuda")
    with torch.cuda.stream(torch.cuda.Stream()):
        with pytest.raises(ValueError):
            layer_norm(ctx, x)


def test_scratch_memory_on_another_stream():
    """The binding's own scratch memory belongs to the context's stream, whichever is current."""
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = HEContext.from_params(config_params(0))
    g = T.rng(4)
    dy, u = torch.randn((3000, 40), generator=g), torch.randn((3000, 70), generator=g)
    codes, exponents = T.keep(u)
    ddy, dc, de, dw = dy.cuda(), R.code_rows(codes), exponents.cuda(), torch.empty((40, 70), device="cuda")
    assert ctx.he_work_weight_grad_q8(3000, 40, 70, torch.float32) > 0
    torch.cuda.synchronize()
    ctx.he_weight_grad_q8(ddy, dc, de, dw)                    # the default stream is the current one
    other = torch.full((1 << 22,), math.nan, device="cuda")   # memory that the scratch must not be taken for
    stream.synchronize()
    kept, d = T.kept(codes, exponents), dy.double()
    near(dw, d.T @ kept, d.abs().T @ kept.abs(), torch.float32, 3016 * 2.0 ** -24)
    assert other.isnan().all()


def test_in_a_graph():
    """All of them captured once, with scratch memory of the graph's own, and replayed on other inputs with eager work between."""
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    rows, dim, hidden, vocab, k = 70, 300, 200, 20000, 6
    g = T.rng(5)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = HEContext.from_params(config_params(0))
        f = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        x, dz, w, c = f(rows, dim), f(rows, hidden), f(dim) + 1, torch.tensor([0.0, 1.0, 0.25, -0.1], device="cuda")
        z, tokens, weights = f(3, vocab), torch.tensor([4, 5, -1], dtype=torch.int32, device="cuda"), f(3) + 0.5
        y, stats, a, codes, exps = f(rows, dim), f(rows, 4), f(rows, dim), f(rows, 304, dtype=torch.uint8)[:, :dim], f(rows, 3, dtype=torch.uint8)
        dw, da, dy, dc, dx, dnw, dnb = f(hidden, dim), f(rows, dim), f(rows, dim), f(4), f(rows, dim), f(dim), f(dim)
        logp, entropy, values, index, lstats, dlogits = f(3), f(3), f(3, k), f(3, k, dtype=torch.int32), f(3, 4), f(3, vocab)

        def run():
            ctx.he_layernorm(x, y, 1e-5, weight=w, stats=stats)
            ctx.he_poly_q8(y, codes, exps, coefs=c, y=a)
            ctx.he_weight_grad_q8(dz, codes, exps, dw)
            ctx.he_poly_grad_q8(codes, exps, c, a, dy, dcoefs=dc)
            ctx.he_layernorm_grad(x, stats, dy, dx, weight=w, dweight=dnw, dbias=dnb)
            ctx.he_token_logprobs(z, 1.0, tokens=tokens, logp=logp, entropy=entropy, values=values, index=index, stats=lstats)
            ctx.he_token_logprobs_grad(z, 1.0, lstats, dlogits, tokens=tokens, logp_weights=weights, entropy_weights=weights)

        outs = (y, a, codes, exps, dw, dy, dc, dx, dnw, dnb, logp, entropy, values, index, dlogits)
        run()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
        for seed in range(4):
            x.copy_(torch.randn((rows, dim), generator=g))
            dz.copy_(torch.randn((rows, hidden), generator=g))
            z.copy_(torch.randn((3, vocab), generator=g))
            graph.replay()
            stream.synchronize()
            got = [t.clone() for t in outs]
            run()
            stream.synchronize()
            for one, two in zip(got, outs):
                assert torch.equal(one, two)


def test_another_current_stream_and_wrong_places(ctx):
    """Tensors that are not on the context's GPU are refused before anything is launched."""
    x = torch.zeros((4, 64))
    with pytest.raises((TypeError, ValueError)):
        ctx.he_layernorm(x, x.clone(), 1e-5)
    with pytest.raises((TypeError, ValueError)):
        ctx.he_layernorm(x.cuda(), x.clone(), 1e-5)
    with pytest.raises((TypeError, ValueError)):
        ctx.he_layernorm_grad(x.cuda(), torch.zeros((4, 4), device="cuda"), x.cuda(), x.cuda(), dweight=torch.zeros(64, device="cuda"), work=torch.zeros(1 << 16))
