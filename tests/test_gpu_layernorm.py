"""GPU: layer norm and its gradients against their definitions in 64 bits.

Tolerances.  A sum in 32 bits of up to 128 numbers one after another, then over the threads, is off by 2^-17 of the sum of their
magnitudes; the mean's lack, the variance and so a normed value n by 2^-17 (1 + |n|).  A gradient by the rows is three terms and two means of
such (up to 256 numbers one after another: 2^-16), the sums over the rows take up to 512 of them: 2^-15 of the terms' magnitudes.  Then one rounding."""
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


def gpu(t):
    return None if t is None else t.cuda()


def run(ctx, x, residual, weight, bias, eps, pitch=None, offset=0, over=None):
    rows, dim = x.shape
    dx, dr = R.on_gpu(x, pitch, offset), None if residual is None else R.on_gpu(residual, pitch, offset)
    total = None if residual is None else R.matrix(rows, dim, x.dtype, pitch, offset)
    y = R.matrix(rows, dim, x.dtype, pitch, offset)
    if over == "x":
        y = dx
    elif over == "both":
        total, y = dx, dr
    stats = torch.empty((rows, 4), device="cuda")
    ctx.he_layernorm(dx, y, eps, weight=gpu(weight), bias=gpu(bias), residual=dr, sum_out=total, stats=stats)
    assert T.untouched(y) and (total is None or T.untouched(total))
    return y, total, stats


def check_forward(got, x, residual, weight, bias, eps):
    y, total, stats = got
    dtype = x.dtype
    h = x if residual is None else (x.float() + residual.float()).to(dtype)
    if residual is not None:
        assert torch.equal(total.cpu(), h)
    n, r = T.norm(h, eps)
    w = torch.ones(1, dtype=torch.float64) if weight is None else weight.double()
    b = torch.zeros(1, dtype=torch.float64) if bias is None else bias.double()
    want = n * w + b
    bound = 2.0 ** -17 * (1 + n.abs()) * w.abs() + 2.0 ** -22 * ((n * w).abs() + b.abs()) + T.rounding(want, dtype)
    off = (y.cpu().double() - want).abs()
    assert (off <= bound).all(), float((off / bound).max())
    s = stats.cpu().double()
    mean, spread = h.double().mean(dim=1), (h.double() - h.double().mean(dim=1, keepdim=True)).abs().mean(dim=1)
    assert ((s[:, 0] + s[:, 1] - mean).abs() <= 2.0 ** -17 * spread + 2.0 ** -46 * mean.abs() + 1e-38).all()
    assert ((s[:, 2] - r[:, 0]).abs() <= 2.0 ** -17 * r[:, 0] + 2.0 ** -149).all() and (s[:, 3] == 0).all()


SHAPES = [(1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (3, 100), (9, 512), (6, 513), (5, 1000), (2, 1025), (3, 2049), (2, 4096), (3, 4099), (2, 8200), (2, 16391), (1, 32768), (2, 65536)]


def inputs(rows, dim, dtype, params, seed, residual=True):
    g = T.rng(seed)
    x = ((torch.randn((rows, dim), generator=g) + 0.7) * torch.exp(0.7 * torch.randn(dim, generator=g))).to(dtype)
    res = (2 * torch.randn((rows, dim), generator=g)).to(dtype) if residual else None
    return x, res, (1 + 0.3 * torch.randn(dim, generator=g)).to(params), (0.2 * torch.randn(dim, generator=g)).to(params)


@pytest.mark.parametrize("rows,dim", SHAPES)
@pytest.mark.parametrize("dtype,params", T.PAIRS)
def test_forward(ctx, dtype, params, rows, dim):
    x, res, w, b = inputs(rows, dim, dtype, params, dim)
    for n, (r_, w_, b_, over) in enumerate(((res, w, b, None), (None, w, None, "x"), (None, None, b, None), (res, None, None, "both"))):
        check_forward(run(ctx, x, r_, w_, b_, 1e-5, dim + n, n, over), x, r_, w_, b_, 1e-5)


@pytest.mark.parametrize("dim,each", [(100, 8), (250, 16), (500, 8), (1000, 16), (2000, 8), (4000, 16), (8000, 16), (16000, 16), (30000, 32), (60000, 64)])
def test_roundings_of_32_bits(ctx, dim, each):
    """A thread adds `each` numbers, then 6 joins in a wavefront and up to 16 of wavefronts: that many roundings and one more of the mean's lack, against the mean of |n|, at most 1; half of them
    and 6 of n, of its size; two of the result."""
    x, _, w, b = inputs(7, dim, torch.float32, torch.float32, dim, False)
    y, _, _ = run(ctx, x, None, w, b, 1e-5)
    n, _ = T.norm(x, 1e-5)
    want = n * w.double() + b.double()
    bound = 2.0 ** -24 * (((each + 24) / 2 + 6) * (n * w).abs() + (each + 23) * w.double().abs() + 2 * ((n * w).abs() + b.double().abs())) + 2.0 ** -149
    off = (y.cpu().double() - want).abs()
    assert (off <= bound).all(), float((off / bound).max())


@pytest.mark.parametrize("dim", [5, 64, 1000, 3000, 20000])
def test_rows_that_are_hard(ctx, dim):
    g = T.rng(dim)
    x = torch.randn((8, dim), generator=g)
    x[0] = 0                                                      # no variance
    x[1] = -3.25
    x[2] += 1e4                                                   # far from 0
    x[3] = x[3] * 1e-3 + 5e5
    x[4] *= 1e30                                                  # squares beyond 32 bits
    x[5] = torch.where(torch.arange(dim) % 2 == 0, 3.2e38, -3.1e38)
    x[6] = 3.3e38                                                 # a sum beyond them
    x[7] *= 1e-6
    w, b = torch.randn(dim, generator=g), torch.randn(dim, generator=g)
    for eps in (1e-5, 0.0, 1e-12):
        y, _, stats = run(ctx, x, None, w, b, eps)
        keep = torch.tensor([i for i in range(8) if i not in (1, 6)])
        check_forward((y[keep.cuda()], None, stats[keep.cuda()]), x[keep], None, w, b, eps)
        # a constant: its mean's rounding is all that is left of it, times 1/sqrt(eps) at most; without eps that may be any n, of size sqrt(dim) at most
        for i in (1, 6):
            c = float(x[i, 0].abs())
            n = ((y[i].cpu().double() - b.double()) / w.double()).abs()
            assert (n <= (min(math.sqrt(dim), 2.0 ** -46 * c * 300 / math.sqrt(eps)) if eps else math.sqrt(dim)) * 1.01 + 1e-4 * (1 + (b / w).abs())).all()


@pytest.mark.parametrize("dim", [100, 1000, 4096, 9000])
def test_rows_whose_spread_is_a_few_roundings(ctx, dim):
    """A mean of 2^20 to 2^24 and numbers that differ by 1 or 2: the rounding of the sum of them is as large as what they differ by."""
    g = T.rng(dim)
    x = 2.0 ** torch.arange(20, 25)[:, None].float() + torch.randint(0, 3, (5, dim), generator=g).float() * torch.tensor([1.0, 1, 1, 1, 2])[:, None]
    w = torch.randn(dim, generator=g)
    check_forward(run(ctx, x, None, w, None, 1e-5), x, None, w, None, 1e-5)
    dy = torch.randn((5, dim), generator=g)
    check_grad(run_grad(ctx, x, 1e-5, dy, w, None, torch.float32), x, 1e-5, dy, w, None, torch.float32)


@pytest.mark.parametrize("dim", [2, 5, 64, 700, 1000, 3000, 5001, 12000, 20000, 40001, 65536])
def test_constant_rows(ctx, dim):
    """No spread, whatever the size: a sum that 32 bits do not hold, or one whose rounding times 1/sqrt(eps) is far from 0."""
    g = T.rng(dim)
    c = torch.tensor([3.3e38, -3.4e38, 2.0 ** 120 * 1.37, 1.1e15, -7.3e27, -3.25, 0.1])
    x, w, b, dy = c[:, None].expand(7, dim).contiguous(), torch.randn(dim, generator=g), torch.randn(dim, generator=g), torch.randn((7, dim), generator=g)
    for eps in (1e-5, 3.0, 1e-12, 0.0):
        y, _, stats = run(ctx, x, None, w, b, eps)
        s, r = stats.cpu().double(), 1 / math.sqrt(float(torch.tensor(eps))) if eps else 0.0
        assert torch.equal(y.cpu(), b.expand(7, dim))
        assert torch.equal(s[:, 0] + s[:, 1], c.double()) and ((s[:, 2] - r).abs() <= 2.0 ** -22 * r).all() and (s[:, 3] == 0).all()
        d = torch.randn((7, dim), generator=g)
        dx, dw, db = run_grad(ctx, x, eps, dy, w, d, torch.float32)
        t = dy.double() * w.double()                          # dx = (g - mean g) / sqrt(eps) + dsum
        mean, size = t.mean(dim=1, keepdim=True), r * (t.abs() + t.abs().mean(dim=1, keepdim=True)) + d.double().abs()
        assert ((dx.cpu().double() - (r * (t - mean) + d.double())).abs() <= 2.0 ** -15 * size + 2.0 ** -149).all()
        assert (dw == 0).all() and ((db.cpu().double() - dy.double().sum(dim=0)).abs() <= 2.0 ** -15 * dy.double().abs().sum(dim=0)).all()


def nearly_constant(dim, size):
    """A constant whose sum rounds alike everywhere, and one element that differs by its last bit: far less than the mean's rounding."""
    c = (torch.tensor([1.2345678, 1.4142135, 1.9999998, 1.0000001]) * size)[:, None].expand(4, dim).contiguous()
    c[:, dim // 3] = torch.nextafter(c[:, 0], c[:, 0] * 2)
    return c


@pytest.mark.parametrize("dim", [50, 900, 5000, 20001])
def test_nearly_constant_rows_whose_sum_leaves_32_bits(ctx, dim):
    x, w = nearly_constant(dim, 2.0 ** 127), torch.randn(dim, generator=T.rng(dim))
    check_forward(run(ctx, x, None, w, None, 1e-5), x, None, w, None, 1e-5)


@pytest.mark.parametrize("dim", [300, 5000, 20001, 32776, 40001, 65536])
def test_nearly_constant_rows(ctx, dim):
    x, w = nearly_constant(dim, 2.0 ** 20), torch.randn(dim, generator=T.rng(dim))
    for eps in (0.0, 1e-5):
        check_forward(run(ctx, x, None, w, None, eps), x, None, w, None, eps)


def test_what_is_not_a_number_stays_in_its_row(ctx):
    x = torch.randn((5, 700), generator=T.rng(1))
    x[1, 3], x[2, 699], x[3, 0] = math.nan, math.inf, -math.inf
    y, _, stats = run(ctx, x, None, None, None, 1e-5)
    assert y[[0, 4]].isfinite().all() and y[1:4].isnan().all() and stats[1:4, 2].isnan().all()


def run_grad(ctx, h, eps, dy, weight, dsum, params, pitch=None, offset=0, over=None, sums="both"):
    rows, dim = h.shape
    d = R.on_gpu(h, pitch, offset)
    stats = torch.empty((rows, 4), device="cuda")
    ctx.he_layernorm(d, torch.empty((rows, dim), dtype=h.dtype, device="cuda"), eps, stats=stats)
    ddy, dds = R.on_gpu(dy, pitch, offset), None if dsum is None else R.on_gpu(dsum, pitch, offset)
    dx = ddy if over == "dy" else dds if over == "dsum" else R.matrix(rows, dim, h.dtype, pitch, offset)
    dw = torch.full((dim,), math.nan, dtype=params, device="cuda") if sums in ("both", "weight") else None
    db = torch.full((dim,), math.nan, dtype=params, device="cuda") if sums in ("both", "bias") else None
    ctx.he_layernorm_grad(d, stats, ddy, dx, weight=gpu(weight), dsum=dds, dweight=dw, dbias=db)
    assert T.untouched(dx)
    return dx, dw, db


def check_grad(got, h, eps, dy, weight, dsum, params):
    dx, dw, db, size, size_w, size_b = T.norm_grad(h, dy, weight, dsum, eps)
    off = (got[0].cpu().double() - dx).abs()
    bound = 2.0 ** -15 * size + T.rounding(dx, h.dtype)
    assert (off <= bound).all(), float((off / bound).max())
    for t, want, s in ((got[1], dw, size_w), (got[2], db, size_b)):
        if t is not None:
            off, bound = (t.cpu().double() - want).abs(), 2.0 ** -15 * s + T.rounding(want, params)
            assert (off <= bound).all(), float((off / bound).max())


@pytest.mark.parametrize("rows,dim", SHAPES + [(700, 33), (1100, 1), (300, 1500), (513, 264)])
@pytest.mark.parametrize("dtype,params", T.PAIRS)
def test_grad(ctx, dtype, params, rows, dim):
    g = T.rng(dim)
    x, ds, w, _ = inputs(rows, dim, dtype, params, dim)
    dy = torch.randn((rows, dim), generator=g).to(dtype)
    for n, (w_, ds_, over, sums) in enumerate(((w, ds, None, "both"), (w, None, "dy", "weight"), (None, ds, "dsum", "bias"), (None, None, None, "none"))):
        check_grad(run_grad(ctx, x, 1e-5, dy, w_, ds_, params, dim + n, n, over, sums), x, 1e-5, dy, w_, ds_, params)


@pytest.mark.parametrize("rows,dim", [(17000, 20), (16500, 200), (1030, 500), (2100, 700), (1100, 1500), (600, 5000), (300, 12001)])
@pytest.mark.parametrize("dtype,params", T.PAIRS[:4:3])
def test_grad_of_more_rows_than_parts(ctx, dtype, params, rows, dim):
    g = T.rng(rows)
    x, ds, w, _ = inputs(rows, dim, dtype, params, dim)
    dy = torch.randn((rows, dim), generator=g).to(dtype)
    for n, (ds_, over) in enumerate(((ds, "dsum"), (None, "dy"), (ds, None))):
        check_grad(run_grad(ctx, x, 1e-5, dy, w, ds_, params, dim + n, n, over), x, 1e-5, dy, w, ds_, params)


def test_grad_of_hard_rows(ctx):
    """Rows far from 0, whose normed values need what the mean lacks; and rows without a variance, which have a gradient by the bias alone."""
    g = T.rng(3)
    x = torch.randn((6, 900), generator=g)
    x[0] += 1e4
    x[1] = 1e-2 * x[1] - 3e3
    x[2] *= 1e25
    x[3] = 0
    dy, w = torch.randn((6, 900), generator=g), torch.randn(900, generator=g)
    for eps in (0.0, 1e-5):
        check_grad(run_grad(ctx, x, eps, dy, w, None, torch.float32), x, eps, dy, w, None, torch.float32)
    got = run_grad(ctx, torch.zeros((4, 50)), 0.0, dy[:4, :50], None, None, torch.float32)
    assert (got[0] == 0).all() and (got[1] == 0).all()


@pytest.mark.parametrize("dim", [5, 20, 200, 500, 900, 1500, 4000, 8000, 12000, 20000])
@pytest.mark.parametrize("dtype,params", T.PAIRS[:2])
def test_grad_of_rows_as_wide_as_their_type(ctx, dtype, params, dim):
    """Differences from the mean that 32 bits do not hold."""
    g = T.rng(dim)
    h, dy, w = torch.full((5, dim), -3e38), torch.randn((5, dim), generator=g).to(dtype), torch.randn(dim, generator=g).to(params)
    h[torch.arange(5), torch.arange(5) * dim // 5] = 3.2e38
    h[3] = -h[3]
    ds = (1e-38 * torch.randn((5, dim), generator=g)).to(dtype)
    for ds_ in (None, ds):
        check_grad(run_grad(ctx, h.to(dtype), 1e-5, dy, w, ds_, params), h.to(dtype), 1e-5, dy, w, ds_, params)


@pytest.mark.parametrize("dim", [1, 5, 7, 13, 300, 5001, 20001])
def test_grad_of_constants_far_out(ctx, dim):
    """A mean times 1/sqrt(eps) that 32 bits do not hold, n being 0 everywhere; statistics as given."""
    g, c, r = T.rng(dim), torch.tensor([3.3e38, -1.1e36, 2.5]), 2.0 ** 10
    dy, w = torch.randn((3, dim), generator=g), torch.randn(dim, generator=g)
    stats = torch.stack([c, torch.zeros(3), torch.full((3,), r), torch.zeros(3)], dim=1).cuda()
    dx, dw = torch.empty((3, dim), device="cuda"), torch.empty(dim, device="cuda")
    ctx.he_layernorm_grad(c[:, None].expand(3, dim).contiguous().cuda(), stats, dy.cuda(), dx, weight=w.cuda(), dweight=dw)
    t = dy.double() * w.double()
    mean, size = t.mean(dim=1, keepdim=True), r * (t.abs() + t.abs().mean(dim=1, keepdim=True))
    assert ((dx.cpu().double() - r * (t - mean)).abs() <= 2.0 ** -15 * size).all() and (dw == 0).all()


def test_gradient_against_differences(ctx):
    """Central differences of sum(y t): the third derivative of a normed row of variance about 1 is below 40 |t|, a value's rounding 2^-17 of its size."""
    rows, dim, h = 2, 9, 2.0 ** -6
    g = T.rng(5)
    x, t, w = torch.randn((rows, dim), generator=g), torch.randn((rows, dim), generator=g), 1 + 0.2 * torch.randn(dim, generator=g)
    dx, _, _ = run_grad(ctx, x, 0.5, t, w, None, torch.float32)
    for j in range(dim):
        up, down = x.clone(), x.clone()
        up[:, j] += h
        down[:, j] -= h
        f = [(run(ctx, v, None, w, None, 0.5)[0].cpu().double() * t).sum(dim=1) for v in (up, down)]
        assert ((f[0] - f[1]) / (2 * h) - dx[:, j].cpu()).abs().max() <= h * h / 6 * 40 * float((t * w).norm()) + 2.0 ** -17 * dim * 4 / h


def test_sums_of_many_rows_with_the_same_bits(ctx):
    """Whole numbers: sums of dy are exact, in any order; the same call gives the same bits."""
    g = T.rng(6)
    x, dy = torch.randn((5000, 130), generator=g), torch.randint(-8, 9, (5000, 130), generator=g).float()
    runs = [run_grad(ctx, x, 1e-5, dy, None, None, torch.float32) for _ in range(3)]
    assert torch.equal(runs[0][2].cpu(), dy.sum(dim=0))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))
    check_grad(runs[0], x, 1e-5, dy, None, None, torch.float32)


def test_far_rows(ctx):
    rows, dim, pitch = 18, 300, 1 << 28                                # 17 * 2^28 elements: past 2^32
    g = T.rng(7)
    x, dy = [torch.randn((rows, dim), generator=g).to(torch.bfloat16) for _ in range(2)]

    def far(t):
        m = torch.empty((rows - 1) * pitch + dim, dtype=t.dtype, device="cuda").as_strided((rows, dim), (pitch, 1))
        return m.copy_(t.cuda())

    stats, y = torch.empty((rows, 4), device="cuda"), far(x)
    ctx.he_layernorm(y, y, 1e-5, stats=stats)
    check_forward((y, None, stats), x, None, None, None, 1e-5)
    y.copy_(x.cuda())
    d, db, dw = far(dy), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    ctx.he_layernorm_grad(y, stats, d, d, dweight=dw, dbias=db)
    check_grad((d, dw, db), x, 1e-5, dy, None, None, torch.float32)


def test_no_rows(ctx):
    e = torch.zeros((0, 40), device="cuda")
    ctx.he_layernorm(e, e.clone(), 1e-5, stats=torch.zeros((0, 4), device="cuda"))
    dw, db = torch.full((40,), math.nan, device="cuda"), torch.full((40,), math.nan, device="cuda")
    ctx.he_layernorm_grad(e, torch.zeros((0, 4), device="cuda"), e, e.clone(), dweight=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()


def test_refusals(ctx):
    from paper_2302_02407_amd.binding import HEError
    x, s = torch.zeros((4, 100), device="cuda"), torch.zeros((4, 4), device="cuda")
    f = lambda *n, **k: torch.zeros(n, device="cuda", **k)  # noqa: E731

    def refused(call, *a, **kw):
        with pytest.raises((HEError, TypeError, ValueError)) as e:
            call(*a, **kw)
        assert not isinstance(e.value, HEError) or e.value.code == -1

    ln, grad = ctx.he_layernorm, ctx.he_layernorm_grad
    refused(ln, x, f(4, 99), 1e-5)
    refused(ln, x, f(4, 100), -1.0)
    refused(ln, x, f(4, 100), math.nan)
    refused(ln, x, f(4, 100), math.inf)
    refused(ln, x, f(4, 100, dtype=torch.bfloat16), 1e-5)
    refused(ln, x.double(), f(4, 100), 1e-5)
    refused(ln, x, f(4, 100), 1e-5, residual=x)                           # without room for the sum
    refused(ln, x, f(4, 100), 1e-5, weight=f(99))
    refused(ln, x, f(4, 100), 1e-5, weight=f(100, dtype=torch.bfloat16))
    refused(ln, x, f(4, 100), 1e-5, weight=f(100), bias=f(100).half())
    refused(ln, x, f(4, 100), 1e-5, stats=f(4, 3))
    refused(ln, x.cpu(), f(4, 100), 1e-5)
    refused(ln, x, x.view(-1)[:400].view(4, 100).expand(4, 100)[:, :].as_strided((4, 100), (99, 1)), 1e-5)     # rows that overlap
    refused(ln, x[:3], x[1:], 1e-5)                                       # onto other rows
    refused(ln, f(4, 65537), f(4, 65537), 1e-5)
    refused(grad, x, s, x.clone(), f(4, 100), dweight=f(100), dbias=f(100, dtype=torch.bfloat16))
    refused(grad, x, s, x.clone(), x, dweight=f(100))                     # onto what is still read
    refused(grad, x, f(3, 4), x.clone(), f(4, 100))
    refused(grad, x, s, x.clone(), f(4, 100), dweight=f(100), work=f(1))  # too little room
    refused(grad, x, s, x.clone(), f(4, 100), dsum=f(4, 99))
    torch.cuda.synchronize()
