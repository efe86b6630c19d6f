"""GPU: the polynomial activation that keeps its input in 8 bits, and its gradients, against their definitions in 64 bits.

Tolerances.  Codes and powers are exact.  A polynomial of up to 9 terms by multiply-adds is off by 2^-19 of the sum of its terms' magnitudes (16 roundings),
a slope times dy by 2^-19 too; a sum over the elements takes products of up to 9 factors and eight terms in 32 bits, 17 roundings: 2^-19 of the
sum of magnitudes.  Then one rounding."""
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


def coefs_of(n, seed=0):
    g = T.rng(seed + n)
    return torch.randn(n, generator=g) / torch.tensor([float(math.factorial(i)) for i in range(n)])


def run(ctx, u, coefs, pitch=None, offset=0, over=False, e8m0=False):
    rows, dim = u.shape
    kb = -(-dim // 128)
    du = R.on_gpu(u, pitch, offset)
    y = None if coefs is None else du if over else R.matrix(rows, dim, u.dtype, pitch, offset)
    codes = R.matrix(rows, dim, R.F8, -(-dim // 16) * 16 + 16)
    room = torch.full((rows, kb + 1), 77, dtype=torch.uint8, device="cuda")
    exponents = room[:, :kb].view(torch.float8_e8m0fnu) if e8m0 else room[:, :kb]
    ctx.he_poly_q8(du, codes, exponents, coefs=None if coefs is None else coefs.cuda(), y=y)
    assert (room[:, kb:] == 77).all() and (y is None or T.untouched(y))
    whole = torch.empty(0, dtype=torch.uint8, device="cuda").set_(codes.untyped_storage())
    assert int((whole != 0x7f).sum()) <= rows * dim                       # what lies around the codes is as it was
    return y, codes, room[:, :kb]


def check(got, u, coefs):
    codes, exponents = T.keep(u.float())
    assert torch.equal(got[2].cpu(), exponents)
    a, b = got[1].cpu().float(), codes.float()
    assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())
    if coefs is not None:
        y, size = T.poly(u, coefs)
        fine = u.isfinite() & (y.to(u.dtype).double() != got[0].cpu().double())      # what the type rounds to an infinity is one
        off, bound = (got[0].cpu().double() - y).abs(), 2.0 ** -19 * size + T.rounding(y, u.dtype)
        assert (off <= bound)[fine].all()


SHAPES = [(1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (3, 127), (9, 128), (6, 129), (5, 1000), (2, 2049), (70, 300), (1, 65536)]


@pytest.mark.parametrize("rows,dim", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_forward(ctx, dtype, rows, dim):
    g = T.rng(dim)
    u = (torch.randn((rows, dim), generator=g) * torch.exp(torch.randn((rows, 1), generator=g))).to(dtype)
    for n, (degree, over) in enumerate(((1, False), (3, True), (0, False), (8, False), (None, False))):
        coefs = None if degree is None else coefs_of(degree + 1)
        check(run(ctx, u, coefs, dim + n, n, over, e8m0=n == 1), u, coefs)


@pytest.mark.parametrize("dtype", TYPES)
def test_blocks_at_the_edges_of_the_powers(ctx, dtype):
    """Every power of two, and 1.75 of it with the numbers on both sides; blocks of zeros, of the least numbers, ties between codes, and what is not finite."""
    most, least = {torch.float32: (127, -149), torch.bfloat16: (127, -133), torch.float16: (15, -24)}[dtype]
    e = torch.arange(least, most + 1).double()
    tops = torch.cat([2.0 ** e, 1.75 * 2.0 ** e]).to(dtype)
    tops = torch.cat([tops, torch.nextafter(tops, tops * 2), torch.nextafter(tops, tops * 0)]) if dtype == torch.float32 else torch.cat([tops, tops * 1.01, tops * 0.99])
    u = tops.double()[:, None] * torch.cat([torch.ones(1), torch.randn(140, generator=T.rng(1)).clamp(-1, 1), torch.arange(1, 60) / 64.0]).double()[None, :]
    u = torch.where(u.abs() > torch.finfo(dtype).max, u.sign() * torch.finfo(dtype).max, u).to(dtype)
    check(run(ctx, u, None), u, None)
    u = torch.randn((8, 300), generator=T.rng(2)).to(dtype)
    u[0], u[1, :128], u[2, 5], u[3, 200], u[4, 299] = 0, 0, math.nan, math.inf, -math.inf
    u[5] = (torch.arange(300) % 17 + 0.5).to(dtype) / 16
    check(run(ctx, u, coefs_of(4)), u, coefs_of(4))


def run_grad(ctx, codes, exponents, coefs, dy, pitch=None, offset=0, over=False, sums=True):
    rows, dim = dy.shape
    dc, ddy = R.code_rows(codes, 1), R.on_gpu(dy, pitch, offset)
    du = ddy if over else R.matrix(rows, dim, dy.dtype, pitch, offset)
    dcoefs = torch.full((len(coefs),), math.nan, device="cuda") if sums else None
    ctx.he_poly_grad_q8(dc, exponents.cuda(), coefs.cuda(), ddy, du, dcoefs=dcoefs)
    assert T.untouched(du)
    return du, dcoefs


def check_grad(got, codes, exponents, coefs, dy):
    du, dc, size, size_c = T.poly_grad(T.kept(codes, exponents), coefs, dy)
    off, bound = (got[0].cpu().double() - du).abs(), 2.0 ** -19 * size + T.rounding(du, dy.dtype)
    assert (off <= bound).all(), float((off / bound).max())
    if got[1] is not None:
        off, bound = (got[1].cpu().double() - dc).abs(), 2.0 ** -19 * size_c + T.rounding(dc, torch.float32)
        assert (off <= bound).all(), float((off / bound).max())


@pytest.mark.parametrize("rows,dim", SHAPES + [(3000, 40)])
@pytest.mark.parametrize("dtype", TYPES)
def test_grad(ctx, dtype, rows, dim):
    g = T.rng(dim + 1)
    codes, exponents = T.keep(torch.randn((rows, dim), generator=g) * 2)
    dy = torch.randn((rows, dim), generator=g).to(dtype)
    for n, (degree, over, sums) in enumerate(((3, False, True), (1, True, True), (0, False, True), (8, False, True), (2, True, False))):
        check_grad(run_grad(ctx, codes, exponents, coefs_of(degree + 1), dy, dim + n, n, over, sums), codes, exponents, coefs_of(degree + 1), dy)


def test_what_is_not_finite_stays_in_its_block(ctx):
    g = T.rng(3)
    u, dy, c = torch.randn((4, 300), generator=g), torch.randn((4, 300), generator=g), coefs_of(4)
    u[1, 130] = math.inf
    codes, exponents = T.keep(u)
    du, dc = run_grad(ctx, codes, exponents, c, dy)
    bad = torch.zeros(4, 300, dtype=torch.bool)
    bad[1, 128:256] = True
    assert torch.equal(du.cpu().isnan(), bad) and dc.cpu()[1:].isnan().all()


def test_gradients_against_differences(ctx):
    """At values that are kept as they are: central differences are off by h^2/6 of a third derivative and by roundings, 2^-19 of the terms over h."""
    h, c = 2.0 ** -7, coefs_of(6)
    codes, exponents = T.keep(torch.arange(-24, 25).float()[None, :] / 16)
    v = T.kept(codes, exponents).float()
    t = torch.randn((1, 49), generator=T.rng(4))
    du, dc = run_grad(ctx, codes, exponents, c, t)
    f = [run(ctx, v + s * h, c)[0].cpu().double() for s in (1, -1)]
    third = sum(i * (i - 1) * (i - 2) * abs(float(c[i])) * 1.6 ** (i - 3) for i in range(3, 6))
    size = float(T.poly(v.abs().max()[None, None], c)[1])
    assert ((t * (f[0] - f[1]) / (2 * h) - du.cpu()).abs() <= t.abs() * (h * h / 6 * third + 2.0 ** -17 * size / h)).all()
    for i in range(6):                                        # the output is linear in the coefficients
        e = torch.zeros(6)
        e[i] = 1
        f = [(run(ctx, v, c + s * e)[0].cpu().double() * t).sum() for s in (1, -1)]
        assert abs((f[0] - f[1]) / 2 - dc[i].cpu()) <= 2.0 ** -16 * 49 * (size + 1.6 ** 5) * float(t.abs().max())


def test_many_rows_with_the_same_bits(ctx):
    """Whole numbers: sums are exact in any order, and du too."""
    g = T.rng(5)
    v, dy = torch.randint(-4, 5, (9000, 130), generator=g).float(), torch.randint(-3, 4, (9000, 130), generator=g).float()
    codes, exponents = T.keep(v)
    c = torch.tensor([1.0, 2.0, -1.0, 3.0])
    runs = [run_grad(ctx, codes, exponents, c, dy) for _ in range(3)]
    du, dc, _, _ = T.poly_grad(v.double(), c, dy)
    assert torch.equal(runs[0][0].cpu().double(), du) and torch.equal(runs[0][1].cpu().double(), dc)
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))


# powers of two of values and gradients: squares above and below what 32 bits hold, dy v^i not; None: padding, a gradient of 0
@pytest.mark.parametrize("value,gradient", [(66, -100), (100, -120), (-74, 110), (100, None)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sums_of_values_whose_squares_32_bits_do_not_hold(ctx, dtype, value, gradient):
    g = T.rng(7)
    v, dy = torch.randn((9, 300), generator=g), torch.randn((9, 300), generator=g)
    v[::2] *= 2.0 ** value
    if gradient is None:
        dy[::2] = 0
    else:
        v, dy = v[::2], dy[::2] * 2.0 ** gradient
    codes, exponents = T.keep(v)
    for n in (2, 3):                                          # slopes of up to two terms: numbers of 32 bits
        check_grad(run_grad(ctx, codes, exponents, coefs_of(n), dy.to(dtype)), codes, exponents, coefs_of(n), dy.to(dtype))


def check_sums(got, codes, exponents, coefs, dy):
    """The coefficients' gradients alone: a slope there need not be a number of 32 bits."""
    _, dc, _, size = T.poly_grad(T.kept(codes, exponents), coefs, dy)
    off, bound = (got[1].cpu().double() - dc).abs(), 2.0 ** -19 * size + T.rounding(dc, torch.float32)
    assert (off <= bound).all(), float((off / bound).max())


@pytest.mark.parametrize("n", [4, 5, 6, 7, 9])
@pytest.mark.parametrize("high", [1, 57, 100, 126])
def test_sums_of_higher_powers_beside_padding(ctx, n, high):
    """Blocks of padding among others, several of them a wavefront's."""
    g = T.rng(n)
    v, dy = torch.randn((40, 300), generator=g), torch.randn((40, 300), generator=g)
    pad = torch.arange(40) % 3 == 1
    v[pad], dy[pad] = v[pad].clamp(-3, 3) * 2.0 ** high, 0.0
    codes, exponents = T.keep(v)
    check_sums(run_grad(ctx, codes, exponents, coefs_of(n), dy), codes, exponents, coefs_of(n), dy)


# on both sides of the powers whose squares are normal numbers
@pytest.mark.parametrize("value,gradient", [(61, -146), (63, -149), (-44, 0), (-46, 0), (-60, 120), (-70, 120)])
def test_sums_of_fourth_powers_far_out(ctx, value, gradient):
    g = T.rng(8)
    v = (1 + torch.rand((9, 300), generator=g) / 2) * (2.0 * torch.randint(0, 2, (9, 300), generator=g) - 1) * 2.0 ** value
    dy = torch.randint(-2 ** 9, 2 ** 9, (9, 300), generator=g).float() * 2.0 ** (gradient if gradient < 0 else gradient - 9)
    codes, exponents = T.keep(v)
    check_sums(run_grad(ctx, codes, exponents, coefs_of(5), dy), codes, exponents, coefs_of(5), dy)


def test_far_rows(ctx):
    rows, dim, pitch = 18, 300, 1 << 28                                # 17 * 2^28 elements: past 2^32
    g = T.rng(6)
    u, dy, c = torch.randn((rows, dim), generator=g).bfloat16(), torch.randn((rows, dim), generator=g).bfloat16(), coefs_of(4)
    far = lambda dtype, cols: torch.empty((rows - 1) * pitch + -(-cols // 16) * 16, dtype=dtype, device="cuda").as_strided((rows, cols), (pitch, 1))  # noqa: E731
    m, codes, exponents = far(torch.bfloat16, dim), far(torch.uint8, dim).view(R.F8), far(torch.uint8, 3)
    m.copy_(u.cuda())
    ctx.he_poly_q8(m, codes, exponents, coefs=c.cuda(), y=m)
    check((m, codes, exponents), u, c)
    m.copy_(dy.cuda())
    dc = torch.empty(4, device="cuda")
    ctx.he_poly_grad_q8(codes, exponents, c.cuda(), m, m, dcoefs=dc)
    check_grad((m, dc), codes.cpu(), exponents.cpu(), c, dy)


def test_no_rows(ctx):
    e, u8 = torch.zeros((0, 40), device="cuda"), lambda n: torch.zeros((0, n), dtype=torch.uint8, device="cuda")  # noqa: E731
    c, dc = coefs_of(3).cuda(), torch.full((3,), math.nan, device="cuda")
    ctx.he_poly_q8(e, u8(48)[:, :40], u8(1), coefs=c, y=e.clone())
    ctx.he_poly_grad_q8(u8(48)[:, :40], u8(1), c, e, e.clone(), dcoefs=dc)
    assert (dc == 0).all()


def test_refusals(ctx):
    from paper_2302_02407_amd.binding import HEError
    f = lambda *n, **k: torch.zeros(n, device="cuda", **k)  # noqa: E731
    u8 = lambda *n: f(*n, dtype=torch.uint8)  # noqa: E731

    def refused(call, *a, **kw):
        with pytest.raises((HEError, TypeError, ValueError)) as e:
            call(*a, **kw)
        assert not isinstance(e.value, HEError) or e.value.code == -1

    fwd, grad = ctx.he_poly_q8, ctx.he_poly_grad_q8
    u, codes, exps = f(4, 96), u8(4, 96), u8(4, 1)
    refused(fwd, u, codes, exps, coefs=f(3))                              # without an output
    refused(fwd, u, codes, exps, y=f(4, 96))                              # without coefficients
    refused(fwd, u, codes, exps, coefs=f(10), y=f(4, 96))
    refused(fwd, u, codes, u8(4, 2))
    refused(fwd, u, codes, f(4, 1))
    refused(fwd, u, f(4, 96), exps)
    refused(fwd, f(4, 97), u8(4, 97), exps)                               # rows of codes that start anywhere
    refused(fwd, u.double(), codes, exps)
    refused(fwd, u, codes, codes[:, :1])                                  # bytes among the codes
    refused(fwd, u, codes, exps, coefs=f(3), y=f(4, 96, dtype=torch.bfloat16))
    refused(fwd, u, codes, exps, coefs=f(3).double(), y=f(4, 96))
    refused(grad, codes, exps, f(10), u, f(4, 96))
    refused(grad, codes, exps, f(0), u, f(4, 96))
    refused(grad, codes, exps, f(3), u, f(4, 95))
    refused(grad, codes, exps, f(3), u, f(4, 96), dcoefs=f(4))
    refused(grad, codes, exps, f(3), u, f(4, 96), dcoefs=f(3), work=u8(8))
    refused(grad, codes[:3], exps, f(3), u, f(4, 96))
    torch.cuda.synchronize()
