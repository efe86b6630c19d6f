"""GPU: log probabilities of given tokens, entropy, alternatives and their gradient, against their definitions in 64 bits.

Tolerances.  Order and indices are exact.  A sum of exponentials in 32 bits is off by at most 1e-5 of itself (an exponential of -d by a few 2^-24 and by
2^-23 of d, terms beyond d = 40 do not count), so a log probability by 1e-5 and 2^-22 of its size; the entropy is a logarithm of such a sum and a
mean of logarithms: 1e-5 (2 + 2 H).  A gradient's terms are probabilities times weights and logarithms, each off by 1e-5 of itself twice; then one rounding."""
import math

import pytest
import torch

import plain_ref as R
import train_ref as T

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ctx():
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    return HEContext.from_params(config_params(0))


def run(ctx, z, tau, tokens, k, pitch=None, offset=0, dz=None):
    rows = z.shape[0]
    f = lambda *n, **kw: torch.full(n, -7, device="cuda", **kw)  # noqa: E731
    out = {"logp": f(rows, dtype=torch.float32) if tokens is not None else None, "entropy": f(rows, dtype=torch.float32),
           "values": f(rows, k, dtype=torch.float32) if k else None, "index": f(rows, k, dtype=torch.int32) if k else None, "stats": f(rows, 4, dtype=torch.float32)}
    ctx.he_token_logprobs(R.on_gpu(z, pitch, offset) if dz is None else dz, tau, tokens=None if tokens is None else tokens.cuda(), **out)
    return out


def near(got, want, scale=1.0):
    got, same = got.cpu().double(), got.cpu().double() == want           # infinities
    return (same | (got.isnan() & want.isnan()) | ((got - want).abs() <= (1e-5 + 2.0 ** -22 * want.abs()) * scale)).all()


def check(out, z, tau, tokens, k):
    logp, p, entropy = T.distribution(z, tau)
    rows, vocab = z.shape
    if tokens is not None:
        there = (tokens >= 0) & (tokens < vocab)
        want = torch.where(there, logp.gather(1, tokens.clamp(0, vocab - 1).long()[:, None])[:, 0], 0.0)
        assert near(out["logp"], want)
    assert ((out["entropy"].cpu().double() - entropy).abs() <= 1e-5 * (2 + 2 * entropy)).all()
    if k:
        index = T.top_order(z, k)
        assert torch.equal(out["index"].cpu().long(), index)
        assert near(out["values"], logp.gather(1, index))
    s = out["stats"].cpu().double()
    none = (logp == -math.inf).all(dim=1)
    assert torch.equal(s[:, 0], torch.where(none, 0.0, z.double().amax(dim=1)))
    total = torch.where(none, 0.0, -logp.amax(dim=1)).exp()
    assert ((s[:, 1] - torch.where(none, 0.0, total)).abs() <= 1e-5 * total).all()
    assert torch.equal(out["stats"][:, 2], out["entropy"]) and (s[:, 3] == 0).all()


VOCABS = [(1, 1), (3, 2), (5, 10), (2, 63), (4, 65), (7, 250), (3, 1000), (2, 1025), (3, 2049), (2, 4099), (2, 9000), (1, 33001), (1, 70003), (40, 300), (1030, 90)]


@pytest.mark.parametrize("rows,vocab", VOCABS)
@pytest.mark.parametrize("dtype", TYPES)
def test_forward(ctx, dtype, rows, vocab):
    g = T.rng(vocab)
    z = (torch.randn((rows, vocab), generator=g) * 3).to(dtype)
    z[0, vocab - vocab // 5:] = -math.inf
    tokens = torch.randint(-1, vocab + 1, (rows,), generator=g, dtype=torch.int32)
    for n, (k, tau) in enumerate(((0, 1.0), (1, 1.0), (min(vocab, 20), 2.0), (min(vocab, 128), 0.6))):
        check(run(ctx, z, tau, tokens if n != 2 else None, k, vocab + n, n), z, tau, tokens if n != 2 else None, k)


def test_outputs_one_by_one(ctx):
    z = torch.randn((6, 5000), generator=T.rng(1)) * 2
    tokens = torch.arange(6, dtype=torch.int32)
    every = run(ctx, z, 1.0, tokens, 9)
    d = z.cuda()
    for names in (("logp",), ("entropy",), ("values", "index"), ("stats",), ("logp", "stats"), ("entropy", "values", "index")):
        out = {n: torch.empty_like(every[n]) for n in names}
        ctx.he_token_logprobs(d, 1.0, tokens=tokens.cuda() if "logp" in names else None, **out)
        for n in names:
            assert torch.equal(out[n], every[n]), n


def hard_rows(vocab, dtype):
    """Rows whose order is where a selection can go wrong."""
    g, i = T.rng(5), torch.arange(vocab).float()
    rows = [torch.zeros(vocab), torch.full((vocab,), -math.inf), i / 64, -i / 64,                           # all equal, nothing, sorted both ways
            torch.randint(0, 3, (vocab,), generator=g).float(), torch.where(i % 2 == 0, 0.0, -0.0),         # few values, both zeros
            torch.where(i < 100, 50.0, torch.randn(vocab, generator=g)),                                    # the top in a row at the front
            torch.where(i >= vocab - 100, 50.0 + i / vocab, torch.randn(vocab, generator=g))]               # ... and at the end
    rows += [torch.where(i % s == 1, 100.0 + torch.randn(vocab, generator=g), torch.randn(vocab, generator=g)) for s in (8, 64, 512, 2048, 4096)]   # all in one lane
    rows += [torch.where((i / s).floor() % 8 == 1, 100.0 + torch.randn(vocab, generator=g), torch.randn(vocab, generator=g)) for s in (8, 512)]
    few = torch.full((vocab,), -math.inf)
    few[[1, vocab - 1]] = torch.tensor([-3.0, 2.0])
    return torch.stack(rows + [few]).to(dtype)


@pytest.mark.parametrize("vocab", [150, 1000, 5000, 40000])
@pytest.mark.parametrize("dtype", TYPES)
def test_hard_rows(ctx, dtype, vocab):
    z = hard_rows(vocab, dtype)
    for k in (1, 7, 128):
        for part in (z, z[:1], z[7:8]):                       # few rows may be cut in parts
            check(run(ctx, part, 1.5, None, k), part, 1.5, None, k)


@pytest.mark.parametrize("vocab", [520, 1000, 1023])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_short_rows(ctx, dtype, vocab):
    """From 1024 rows on a wavefront takes one of up to 4 KB; k above 32 four."""
    few = hard_rows(vocab, dtype)
    few = torch.cat([few, torch.randn((53, vocab), generator=T.rng(vocab)).to(dtype)])
    z = few.repeat(16, 1)
    logp, _, entropy = T.distribution(few, 1.5)
    index = T.top_order(few, 40)
    for k in (1, 32, 40):
        out = run(ctx, z, 1.5, None, k, vocab + 1, 1)
        assert torch.equal(out["index"].cpu().long(), index[:, :k].repeat(16, 1))
        assert near(out["values"], logp.gather(1, index[:, :k]).repeat(16, 1))
        assert ((out["entropy"].cpu().double() - entropy.repeat(16)).abs() <= 1e-5 * (2 + 2 * entropy.repeat(16))).all()


@pytest.mark.parametrize("rows", [1, 3])
def test_a_large_vocabulary(ctx, rows):
    """2^20 logits, the largest; order compared with a sort."""
    z = torch.randn((rows, 1 << 20), generator=T.rng(6)) * 2
    tokens = torch.full((rows,), (1 << 20) - 1, dtype=torch.int32)
    out = run(ctx, z, 1.0, tokens, 128)
    v, i = z.sort(dim=1, descending=True, stable=True)
    logp, _, entropy = T.distribution(z, 1.0)
    assert torch.equal(out["index"].cpu().long(), i[:, :128]) and near(out["values"], logp.gather(1, i[:, :128])) and near(out["logp"], logp[:, -1])
    assert ((out["entropy"].cpu().double() - entropy).abs() <= 1e-5 * (2 + 2 * entropy)).all()


LOWS = [(torch.float32, torch.finfo(torch.float32).min), (torch.float32, -1e38), (torch.bfloat16, torch.finfo(torch.bfloat16).min), (torch.bfloat16, -3.0e38)]


@pytest.mark.parametrize("vocab", [3, 700, 9001, 40000])
@pytest.mark.parametrize("tau", [0.25, 1.0, 3.0])
@pytest.mark.parametrize("dtype,low", LOWS)
def test_masks_of_the_lowest_value(ctx, vocab, tau, dtype, low):
    """As if they were -infinity, in every sum and gradient; the order takes them as they are."""
    rows, g = 8, T.rng(vocab)
    z = 3 * torch.randn((rows, vocab), generator=g)
    z[0::4][torch.rand((2, vocab), generator=g) < 0.7] = low
    z[1::4] = torch.where((torch.arange(vocab) == 1) | (torch.arange(vocab) == vocab - 1), z[1::4], low)
    z[2::4] = low
    z = z.to(dtype)
    tokens = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    out = run(ctx, z, tau, tokens, min(vocab, 5))
    logp, _, entropy = T.distribution(z, tau)
    assert near(out["logp"], logp.gather(1, tokens.long()[:, None])[:, 0])
    assert ((out["entropy"].cpu().double() - entropy).abs() <= 1e-5 * (2 + 2 * entropy)).all()
    index = T.top_order(z, min(vocab, 5))
    assert torch.equal(out["index"].cpu().long(), index) and near(out["values"], logp.gather(1, index))
    a, b = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    grad = run_grad(ctx, z, tau, tokens, a, b, out["stats"])
    check_grad(grad, z, tau, tokens, a, b)
    assert (grad[2::4] == 0).all()


def test_rows_without_a_distribution(ctx):
    for vocab in (9, 700, 20000):
        z = torch.randn((6, vocab), generator=T.rng(vocab))
        z[1, vocab // 2], z[2, 5], z[3, 1], z[3, 2] = math.nan, math.inf, math.inf, math.inf
        z[4, 3] = 3.3e38
        tokens = torch.tensor([0, 1, 5, 1, 3, -1], dtype=torch.int32)
        out = run(ctx, z, 0.5, tokens, 4)
        bad = torch.tensor([False, True, True, True, True, False])
        for n in ("logp", "entropy"):
            assert torch.equal(out[n].cpu().isnan(), bad)
        assert torch.equal(out["values"].cpu().isnan(), bad[:, None].expand(6, 4)) and torch.equal(out["index"].cpu().long(), T.top_order(z, 4))
        w = torch.tensor([1.0, 1.0, 0.0, 1.0, 1.0, 1.0])
        grad = run_grad(ctx, z, 0.5, tokens, w, None, out["stats"])
        assert grad[0].isfinite().all() and (grad[2] == 0).all() and (grad[5] == 0).all() and grad[[1, 3, 4]].isnan().any(dim=1).all()


def test_logits_far_from_zero(ctx):
    g = T.rng(9)
    z = torch.randn((5, 3000), generator=g) + torch.tensor([0.0, 1e4, -1e4, 1e6, -1e9])[:, None]
    tokens = torch.tensor([5, 6, 7, 8, 9], dtype=torch.int32)
    check(run(ctx, z, 1.0, tokens, 3), z, 1.0, tokens, 3)


def run_grad(ctx, z, tau, tokens, a, b, stats, pitch=None, offset=0, over=False):
    dz = R.on_gpu(z, pitch, offset)
    grad = dz if over else R.matrix(*z.shape, z.dtype, pitch, offset)
    ctx.he_token_logprobs_grad(dz, tau, stats, grad, tokens=None if tokens is None else tokens.cuda(), logp_weights=None if a is None else a.cuda(),
                               entropy_weights=None if b is None else b.cuda())
    assert T.untouched(grad)
    return grad.cpu()


def check_grad(grad, z, tau, tokens, a, b):
    want, size = T.logprobs_grad(z, tau, tokens, a, b)
    bound = 2e-5 * size + T.rounding(want, z.dtype) + 2.0 ** -126
    off = (grad.double() - want).abs()
    assert (off <= bound).all(), float((off / bound).max())


@pytest.mark.parametrize("rows,vocab", VOCABS)
@pytest.mark.parametrize("dtype", TYPES)
def test_grad(ctx, dtype, rows, vocab):
    g = T.rng(vocab + 1)
    z = (torch.randn((rows, vocab), generator=g) * 3).to(dtype)
    z[0, vocab - vocab // 5:] = -math.inf
    tokens = torch.randint(-1, vocab + 1, (rows,), generator=g, dtype=torch.int32)
    a, b = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    a[rows // 2] = 0
    for n, (tau, t, wa, wb, over) in enumerate(((1.0, tokens, a, b, False), (2.0, tokens, a, None, True), (0.6, None, None, b, False), (1.0, tokens, None, None, False))):
        stats = run(ctx, z, tau, None, 0)["stats"]
        check_grad(run_grad(ctx, z, tau, t, wa, wb, stats, vocab + n, n, over), z, tau, t, wa, wb)


def test_gradient_against_differences(ctx):
    """Central differences, h = 2^-4 on logits of size 1: off by h^2/6 of a third derivative (of log p and of the entropy below 2 tau^-3) and by roundings, 1e-4 / h."""
    rows, vocab, tau, h = 3, 12, 2.0, 2.0 ** -4
    g = T.rng(2)
    z, tokens = torch.randn((rows, vocab), generator=g), torch.tensor([3, 0, 11], dtype=torch.int32)
    a, b = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    grad = run_grad(ctx, z, tau, tokens, a, b, run(ctx, z, tau, None, 0)["stats"])
    for j in range(vocab):
        f = []
        for s in (h, -h):
            x = z.clone()
            x[:, j] += s
            out = run(ctx, x, tau, tokens, 0)
            f.append(a * out["logp"].cpu() + b * out["entropy"].cpu())
        assert (((f[0] - f[1]) / (2 * h) - grad[:, j]).abs() <= (a.abs() + b.abs()) * (h * h / 6 * 2 / tau ** 3 + 1e-4 / h)).all()


@pytest.mark.parametrize("rows,vocab", [(40, 20000), (1, 100000)])
def test_the_same_call_gives_the_same_bits(ctx, rows, vocab):
    z = (torch.randn((rows, vocab), generator=T.rng(13)) * 3).bfloat16()
    tokens = torch.arange(rows, dtype=torch.int32)
    runs = [run(ctx, z, 1.0, tokens, 30) for _ in range(3)]
    for r in runs[1:]:
        assert all(torch.equal(r[n], runs[0][n]) for n in r)


def test_far_rows(ctx):
    rows, vocab, pitch = 18, 1000, 1 << 28                        # 17 * 2^28 elements: past 2^32
    z = torch.randn((rows, vocab), generator=T.rng(1)).bfloat16()
    m = torch.empty((rows - 1) * pitch + vocab, dtype=torch.bfloat16, device="cuda").as_strided((rows, vocab), (pitch, 1)).copy_(z.cuda())
    tokens = torch.arange(rows, dtype=torch.int32)
    out = run(ctx, z, 1.5, tokens, 8, dz=m)
    check(out, z, 1.5, tokens, 8)
    a = torch.randn(rows, generator=T.rng(2))
    ctx.he_token_logprobs_grad(m, 1.5, out["stats"], m, tokens=tokens.cuda(), logp_weights=a.cuda())
    check_grad(m.cpu(), z, 1.5, tokens, a, None)


def test_no_rows(ctx):
    f, i32 = torch.zeros((0,), device="cuda"), torch.zeros((0,), dtype=torch.int32, device="cuda")
    ctx.he_token_logprobs(torch.zeros((0, 40), device="cuda"), 1.0, tokens=i32, logp=f, entropy=f.clone())
    ctx.he_token_logprobs_grad(torch.zeros((0, 40), device="cuda"), 1.0, torch.zeros((0, 4), device="cuda"), torch.zeros((0, 40), device="cuda"), tokens=i32, logp_weights=f)


def test_refusals(ctx):
    from paper_2302_02407_amd.binding import HEError
    f = lambda *n, **k: torch.zeros(n, device="cuda", **k)  # noqa: E731
    i32 = lambda *n: f(*n, dtype=torch.int32)  # noqa: E731

    def refused(call, *a, **kw):
        with pytest.raises((HEError, TypeError, ValueError)) as e:
            call(*a, **kw)
        assert not isinstance(e.value, HEError) or e.value.code == -1

    fwd, grad, z = ctx.he_token_logprobs, ctx.he_token_logprobs_grad, f(4, 100)
    refused(fwd, z)                                                       # nothing asked for
    refused(fwd, z, 0.0, entropy=f(4))
    refused(fwd, z, math.nan, entropy=f(4))
    refused(fwd, z, 1.0, logp=f(4))                                       # without tokens
    refused(fwd, z, 1.0, tokens=i32(4), entropy=f(4))
    refused(fwd, z, 1.0, tokens=i32(4).long(), logp=f(4))
    refused(fwd, z, 1.0, tokens=i32(3), logp=f(4))
    refused(fwd, z, 1.0, values=f(4, 5))
    refused(fwd, z, 1.0, index=i32(4, 5), entropy=f(4))
    refused(fwd, z, 1.0, values=f(4, 101), index=i32(4, 101))
    refused(fwd, f(4, 300), 1.0, values=f(4, 129), index=i32(4, 129))
    refused(fwd, z, 1.0, entropy=z.view(-1)[:4])
    refused(fwd, z.double(), 1.0, entropy=f(4))
    refused(fwd, z[:1].expand(4, 100), 1.0, entropy=f(4))
    refused(fwd, f(4, 200)[:, ::2], 1.0, entropy=f(4))
    refused(grad, z, 1.0, f(4, 4), f(4, 99))
    refused(grad, z, 1.0, f(4, 3), f(4, 100))
    refused(grad, z, 1.0, f(4, 4), f(4, 100), logp_weights=f(4))          # without tokens
    refused(grad, z, 1.0, f(4, 4), f(4, 100, dtype=torch.bfloat16))
    room = f(5, 100)
    refused(grad, room[:4], 1.0, f(4, 4), room[1:], entropy_weights=f(4))
    torch.cuda.synchronize()
