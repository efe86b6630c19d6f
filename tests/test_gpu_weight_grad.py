"""GPU: a linear layer's weight gradient from its input as kept in 8 bits, against 64 bits.

Tolerances.  Products are exact; a sum of m of them in 32 bits, in any order, is off by (m + 16) 2^-24 of the sum of their magnitudes.  Then one
rounding, two where it is added to what is there.  With whole numbers everything is exact."""
import math

import pytest
import torch

import plain_ref as R
import train_ref as T

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
OUTS = {torch.float32: [torch.float32], torch.bfloat16: [torch.bfloat16, torch.float32], torch.float16: [torch.float16, torch.float32]}


@pytest.fixture(scope="module")
def ctx():
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    return HEContext.from_params(config_params(0))


def run(ctx, dy, codes, exponents, out, pitch=0, offset=0, onto=None):
    (m, n), k = dy.shape, codes.shape[1]
    dw = R.matrix(n, k, out, k + pitch, offset)
    if onto is not None:
        dw.copy_(onto.cuda())
    e = torch.full((m, exponents.shape[1] + 1), 255, dtype=torch.uint8, device="cuda")[:, :exponents.shape[1]].copy_(exponents.cuda())
    ctx.he_weight_grad_q8(R.on_gpu(dy, n + pitch, offset), R.code_rows(codes, 1 if pitch else 0), e, dw, accumulate=onto is not None)
    assert T.untouched(dw)
    return dw.cpu()


def check(got, dy, codes, exponents, onto=None):
    v, d = T.kept(codes, exponents), dy.double()
    want, size = d.T @ v, d.abs().T @ v.abs()
    if onto is not None:
        want = want + onto.double()
    bound = (dy.shape[0] + 16) * 2.0 ** -24 * size + T.rounding(want, got.dtype) + want.abs() * 2.0 ** -24
    off = (got.double() - want).abs()
    assert (off <= bound).all(), float((off / bound).max())


SHAPES = [(1, 1, 1), (2, 3, 5), (5, 130, 9), (31, 20, 129), (32, 128, 128), (33, 129, 127), (70, 200, 300), (257, 65, 1000), (600, 17, 33), (1000, 300, 16), (2100, 40, 100), (64, 513, 260)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_weight_grad(ctx, dtype, m, n, k):
    g = T.rng(m + n + k)
    codes, exponents = T.keep(torch.randn((m, k), generator=g) * torch.exp(torch.randn((m, 1), generator=g)))
    dy = (torch.randn((m, n), generator=g) * torch.exp(torch.randn((m, 1), generator=g))).to(dtype)
    for i, out in enumerate(OUTS[dtype]):
        check(run(ctx, dy, codes, exponents, out, 3 * i, i), dy, codes, exponents)
    onto = torch.randn((n, k), generator=g).to(out)
    check(run(ctx, dy, codes, exponents, out, 1, 1, onto), dy, codes, exponents, onto)


# tiles of 64 by 256: one and several, ends of both sides, sums in one part and in many
@pytest.mark.parametrize("m,n,k", [(40, 64, 256), (33, 63, 257), (700, 1, 1000), (65, 7, 513), (300, 9, 255), (5000, 33, 700), (20000, 64, 130), (9000, 65, 260)])
@pytest.mark.parametrize("dtype", TYPES)
def test_few_columns(ctx, dtype, m, n, k):
    g = T.rng(m + n + k)
    codes, exponents = T.keep(torch.randn((m, k), generator=g) * torch.exp(torch.randn((m, 1), generator=g)))
    dy = torch.randn((m, n), generator=g).to(dtype)
    check(run(ctx, dy, codes, exponents, torch.float32, 5, 3), dy, codes, exponents)


@pytest.mark.parametrize("m,n,k", [(40, 50, 60), (500, 260, 257), (3000, 130, 70), (9000, 20, 20)])
@pytest.mark.parametrize("dtype", TYPES)
def test_whole_numbers_are_exact(ctx, dtype, m, n, k):
    """dy of up to 11 bits (8 in bfloat16), sums below 2^24."""
    g = T.rng(m)
    most = {torch.float32: 2047, torch.float16: 2047, torch.bfloat16: 255}[dtype] if m < 1000 else 100
    dy, v = torch.randint(-most, most + 1, (m, n), generator=g).to(dtype), torch.randint(-8, 9, (m, k), generator=g).float()
    codes, exponents = T.keep(v)
    exponents[::3] += 1                                                   # each row by a power of its own
    want = dy.double().T @ T.kept(codes, exponents)
    assert torch.equal(run(ctx, dy, codes, exponents, torch.float32).double(), want)


@pytest.mark.parametrize("m,n,k", [(70, 4100, 2900), (33, 3585, 3590), (31, 250, 70000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_whole_numbers_of_large_gradients(ctx, dtype, m, n, k):
    """Enough results for the largest tiles, the last of which begin earlier than where they are counted."""
    g = T.rng(n)
    dy, v = torch.randint(-100, 101, (m, n), generator=g).to(dtype), torch.randint(-8, 9, (m, k), generator=g).float()
    codes, exponents = T.keep(v)
    exponents[::3] += 1
    kept = T.kept(codes, exponents).float()
    want = dy.float().T @ kept                                            # whole numbers below 2^24: exact
    assert torch.equal(run(ctx, dy, codes, exponents, torch.float32, 1, 1), want)
    onto = torch.randint(-100, 101, (n, k), generator=g).float()
    assert torch.equal(run(ctx, dy, codes, exponents, torch.float32, 0, 0, onto), want + onto)


@pytest.mark.parametrize("m,n,k", [(20011, 777, 1001), (2069, 4050, 4060)])
@pytest.mark.parametrize("dtype", TYPES)
def test_whole_numbers_of_long_sums_in_large_tiles(ctx, dtype, m, n, k):
    """Many steps a tile, in parts (40 steps each, 26 the last) and whole (65): sums below m * 20 * 16 < 2^24."""
    g = T.rng(m)
    dy, v = torch.randint(-20, 21, (m, n), generator=g).to(dtype), torch.randint(-8, 9, (m, k), generator=g).float()
    codes, exponents = T.keep(v)
    exponents[::3] += 1
    want = dy.float().T @ T.kept(codes, exponents).float()
    assert torch.equal(run(ctx, dy, codes, exponents, torch.float32, 1, 1), want)


# m, n, k, and of bfloat16 the tile's columns of dy, the parts of the sum, whether rows are asked for further ahead: test_train_checks compares these with the cut
LAUNCHES = [(1000, 10, 40000, 64, 4, 0), (2048, 100, 40000, 128, 2, 0), (4096, 2048, 2048, 128, 3, 0), (1000, 200, 40000, 128, 1, 0), (40, 100, 100000, 128, 1, 0), (70, 50, 40000, 64, 1, 1),
            (70, 100, 40000, 128, 1, 1), (5000, 33, 700, 64, 32, 1), (3000, 130, 70, 128, 16, 1), (9000, 65, 260, 128, 57, 1), (2069, 4050, 4060, 256, 1, 1), (20011, 777, 1001, 256, 16, 1)]


@pytest.mark.parametrize("m,n,k", [row[:3] for row in LAUNCHES])
@pytest.mark.parametrize("dtype", TYPES)
def test_whole_numbers_by_every_launch(ctx, dtype, m, n, k):
    """Sums below m * 20 * 16 < 2^24: exact."""
    g = torch.Generator("cuda").manual_seed(m + n)
    dy = torch.randint(-20, 21, (m, n), generator=g, device="cuda").to(dtype)
    v, exponents = torch.randint(-8, 9, (m, k), generator=g, device="cuda").float(), torch.full((m, -(-k // 128)), 127, dtype=torch.uint8, device="cuda")
    codes = v.to(R.F8)
    exponents[::3] += 1
    v[::3] *= 2
    want = (dy.double().T @ v.double()).float().cpu()
    assert torch.equal(run(ctx, dy, codes, exponents, torch.float32, 1, 1), want)


def test_numbers_of_all_sizes(ctx):
    """32 bits of dy count, far powers of what is kept too: one product a sum, which is added up from three parts of it, so off by at most 3 2^-24 of itself
    and by what is below the smallest normal numbers; what 32 bits do not hold is infinite."""
    g, m = T.rng(1), 96
    dy = torch.diag(torch.randn(m, generator=g) * 2.0 ** torch.randint(-90, 91, (m,), generator=g).float())
    dy[5, 5] = torch.finfo(torch.float32).max
    codes, exponents = T.keep(torch.randn((m, 200), generator=g) * 2.0 ** torch.randint(-30, 31, (m, 1), generator=g).float())
    exponents[5] = 120
    got, want = run(ctx, dy, codes, exponents, torch.float32).double(), dy.double().T @ T.kept(codes, exponents)
    assert (((got - want).abs() <= want.abs() * 3 * 2.0 ** -24 + 2.0 ** -126) | (got == want.float().double())).all()


def test_what_is_not_finite_stays_in_its_row_and_column(ctx):
    g = T.rng(2)
    dy, u = torch.randn((50, 40), generator=g), torch.randn((50, 300), generator=g).abs() + 0.1
    for dtype in TYPES:
        half = dy.to(dtype, copy=True)
        half[7, 3], half[8, 4], half[9, 5] = math.inf, math.nan, -math.inf
        got = run(ctx, half, *T.keep(u), torch.float32)
        assert (got[3] == math.inf).all() and got[4].isnan().all() and (got[5] == -math.inf).all() and got[6:].isfinite().all()
    dy[7, 3], dy[8, 4], u[9, 200] = math.inf, math.nan, math.nan
    codes, exponents = T.keep(u)
    got = run(ctx, dy, codes, exponents, torch.float32)
    bad = torch.zeros(40, 300, dtype=torch.bool)
    bad[[3, 4]], bad[:, 128:256] = True, True
    assert torch.equal(~got.isfinite(), bad) and (got[3, :128] == math.inf).all()


def test_every_f16_nan_stays_one(ctx):
    """Whichever of its bits are set, the lowest three alone too."""
    bits = torch.tensor([0x7c01, 0x7c02, 0x7c04, 0x7c07, 0x7c08, 0x7e00, 0x7fff]).repeat(2) - torch.tensor([0] * 7 + [0x8000] * 7)
    dy = torch.randn((20, 16), generator=T.rng(8)).half()
    for n, b in enumerate(bits.tolist()):
        dy[n, n:n + 1].view(torch.int16).fill_(b)
    assert dy.isnan().sum() == 14
    codes, exponents = T.keep(torch.randn((20, 300), generator=T.rng(9)).abs() + 0.1)
    got = run(ctx, dy, codes, exponents, torch.float32)
    assert got[:14].isnan().all() and got[14:].isfinite().all()


@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_beside_large_powers(ctx, dtype):
    """An infinity times any kept value but 0 is an infinity of the product's sign."""
    dy, v = torch.zeros((20, 16), dtype=dtype), torch.randn((20, 300), generator=T.rng(10))
    v = (v + v.sign()) * 2.0 ** torch.arange(29, 129, 5)[:, None].float()
    for n in range(16):
        dy[n + 4, n] = -math.inf if n % 2 else math.inf
    codes, exponents = T.keep(v)
    got = run(ctx, dy, codes, exponents, torch.float32)
    for n in range(16):
        assert torch.equal(got[n], v[n + 4] * float(dy[n + 4, n]))


def test_a_block_marked_as_not_finite_is_none_whatever_its_codes(ctx):
    codes, exponents = T.keep(torch.randn((40, 300), generator=T.rng(7)))
    exponents[11, 1] = 255
    for dtype in TYPES:
        got = run(ctx, torch.ones((40, 20), dtype=dtype), codes, exponents, torch.float32)
        assert torch.equal(got.isnan(), (torch.arange(300) // 128 == 1).expand(20, 300)) and got[:, :128].isfinite().all()


def test_long_sums_with_the_same_bits(ctx):
    g = T.rng(3)
    codes, exponents = T.keep(torch.randn((20000, 70), generator=g))
    dy = torch.randn((20000, 90), generator=g).bfloat16()
    runs = [run(ctx, dy, codes, exponents, torch.float32) for _ in range(3)]
    check(runs[0], dy, codes, exponents)
    assert all(torch.equal(r, runs[0]) for r in runs[1:])


def test_far_rows(ctx):
    """Whole numbers, rows so far apart that offsets pass 32 bits."""
    g, m, n, k, pitch = T.rng(4), 40, 30, 50, 1 << 27
    far = lambda rows, cols, dtype: torch.empty((rows - 1) * pitch + -(-cols // 16) * 16, dtype=dtype, device="cuda").as_strided((rows, cols), (pitch, 1))  # noqa: E731
    codes, exponents = T.keep(torch.randint(-8, 9, (m, k), generator=g).float())
    dy = torch.randint(-9, 10, (m, n), generator=g).bfloat16()
    dc, de, dd, dw = far(m, k, torch.uint8).view(R.F8), far(m, 1, torch.uint8), far(m, n, torch.bfloat16), far(n, k, torch.float16)
    for a, b in ((dc, codes), (de, exponents), (dd, dy)):
        a.copy_(b.cuda())
    ctx.he_weight_grad_q8(dd, dc, de, dw)
    assert torch.equal(dw.cpu().double(), dy.double().T @ T.kept(codes, exponents))


def test_no_rows(ctx):
    u8 = lambda n: torch.zeros((0, n), dtype=torch.uint8, device="cuda")  # noqa: E731
    dw = torch.full((5, 7), math.nan, device="cuda")
    ctx.he_weight_grad_q8(torch.zeros((0, 5), device="cuda"), u8(16)[:, :7], u8(1), dw)
    assert (dw == 0).all()
    dw.fill_(3)
    ctx.he_weight_grad_q8(torch.zeros((0, 5), device="cuda"), u8(16)[:, :7], u8(1), dw, accumulate=True)
    assert (dw == 3).all()


def test_refusals(ctx):
    from paper_2302_02407_amd.binding import HEError
    f = lambda *n, **k: torch.zeros(n, device="cuda", **k)  # noqa: E731
    u8 = lambda *n: f(*n, dtype=torch.uint8)  # noqa: E731

    def refused(*a, **kw):
        with pytest.raises((HEError, TypeError, ValueError)) as e:
            ctx.he_weight_grad_q8(*a, **kw)
        assert not isinstance(e.value, HEError) or e.value.code == -1

    dy, codes, exps, dw = f(6, 20), u8(6, 32), u8(6, 1), f(20, 32)
    refused(dy, codes, exps, f(20, 31))
    refused(dy, codes, exps, f(32, 20))
    refused(dy[:5], codes, exps, dw)
    refused(dy, codes, u8(6, 2), dw)
    refused(dy, codes, f(6, 1), dw)
    refused(dy.double(), codes, exps, dw)
    refused(dy, codes, exps, dw.double())
    refused(dy, u8(6, 33), u8(6, 1), f(20, 33))                           # rows of codes that start anywhere
    refused(dy, codes, exps, None)
    room = f(6 * 20 + 20 * 32)
    refused(room[:120].view(6, 20), codes, exps, room[100:740].view(20, 32))
    big = u8(40000, 16)
    refused(f(40000, 5), big, u8(40000, 1), f(5, 16), work=u8(16))
    torch.cuda.synchronize()
