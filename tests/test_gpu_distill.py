"""GPU: a row's top logits and the distillation loss with its gradient, against their definitions in 64 bits.

Tolerances.  Values and indices are exact.  A logarithm of a sum of exponentials in 32 bits: an exponential of -d is off by a few
2^-24 and by 2^-23 of d, and terms beyond d = 40 do not count: at most 1e-5 relative, so 1e-5 in the logarithm, and 2^-22 of its
size.  A loss is a mean of such logarithms: 1e-5 of tau^2 (1 - alpha) (1 + its size) and of alpha (1 + ...).  A gradient is a sum of
probabilities, each off by 1e-5 of itself twice, then rounded to its type."""
import math

import pytest
import torch

import plain_ref as R

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ctx():
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    return HEContext.from_params(config_params(0))


def rng(seed):
    return torch.Generator().manual_seed(seed)


def run_top(ctx, z, k, tau, pitch=None, offset=0, rest=True):
    rows = z.shape[0]
    v, i = torch.empty((rows, k), device="cuda"), torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
    r = torch.empty(rows, device="cuda") if rest else None
    ctx.he_top_logits(R.on_gpu(z, pitch, offset), tau, v, i, r)
    return v.cpu().double(), i.cpu().long(), r.cpu().double() if rest else None


def check_top(got, want):
    assert torch.equal(got[1], want[1])
    assert torch.equal(got[0].nan_to_num(nan=1e300), want[0].nan_to_num(nan=1e300))
    same = got[2] == want[2]                       # infinities
    assert (same | (got[2].isnan() & want[2].isnan()) | ((got[2] - want[2]).abs() <= 1e-5 + 2.0 ** -22 * want[2].abs())).all()


@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (5, 10), (2, 63), (4, 65), (7, 250), (3, 1000), (2, 1024), (2, 1025), (3, 2049), (2, 4099), (2, 9000), (1, 33001), (1, 70003)])
@pytest.mark.parametrize("dtype", TYPES)
def test_top(ctx, dtype, rows, vocab):
    g = rng(vocab)
    z = (torch.randn((rows, vocab), generator=g) * 3).to(dtype)
    z[0, vocab - vocab // 5:] = -math.inf
    for k, tau, more, off in ((1, 1.0, 0, 0), (min(vocab, 20), 2.0, 1, 1), (min(vocab, 64), 0.7, 3, 5), (min(vocab, 128), 4.0, 8, 0)):
        check_top(run_top(ctx, z, k, tau, vocab + more, off), R.top(z, k, tau))


def hard_rows(vocab, dtype):
    """Rows whose order is where a selection can go wrong."""
    g, i = rng(5), torch.arange(vocab).float()
    rows = [torch.zeros(vocab), torch.full((vocab,), -math.inf), i / 64, -i / 64,                           # all equal, nothing, sorted both ways
            torch.randint(0, 3, (vocab,), generator=g).float(), torch.where(i % 2 == 0, 0.0, -0.0),         # few values, both zeros
            torch.where(i < 100, 50.0, torch.randn(vocab, generator=g)),                                    # the top in a row at the front
            torch.where(i >= vocab - 100, 50.0 + i / vocab, torch.randn(vocab, generator=g))]               # ... and at the end
    rows += [torch.where(i % s == 1, 100.0 + torch.randn(vocab, generator=g), torch.randn(vocab, generator=g)) for s in (8, 64, 256, 512, 1024, 2048, 4096)]   # all in one lane
    rows += [torch.where((i / s).floor() % 8 == 1, 100.0 + torch.randn(vocab, generator=g), torch.randn(vocab, generator=g)) for s in (8, 64, 512)]
    some = torch.randn(vocab, generator=g)
    some[vocab // 2], some[vocab // 3] = math.inf, -math.inf
    few = torch.full((vocab,), -math.inf)
    few[[1, vocab - 1]] = torch.tensor([-3.0, 2.0])
    nan = torch.randn(vocab, generator=g)
    nan[[3, vocab - 2]] = math.nan
    return torch.stack(rows + [some, few, nan]).to(dtype)


@pytest.mark.parametrize("vocab", [150, 1000, 5000, 20000])
@pytest.mark.parametrize("dtype", TYPES)
def test_top_of_hard_rows(ctx, dtype, vocab):
    z = hard_rows(vocab, dtype)
    for k in (1, 7, 64, 128):
        check_top(run_top(ctx, z, k, 1.5), R.top(z, k, 1.5))


def test_top_of_a_large_vocabulary(ctx):
    """2^20 logits, the largest; the top compared with a sort, the rest with 64 bits."""
    z = torch.randn((2, 1 << 20), generator=rng(6)) * 2
    got = run_top(ctx, z, 128, 2.0)
    v, i = z.double().sort(dim=1, descending=True, stable=True)
    assert torch.equal(got[0], v[:, :128]) and torch.equal(got[1], i[:, :128])
    assert ((got[2] - torch.logsumexp(v[:, 128:] / 2, dim=1)).abs() <= 2e-5).all()
    assert run_top(ctx, z, 5, 2.0, rest=False)[2] is None


def teacher(z, k, tau, g, rest=True):
    t = 0.8 * z.float() + torch.randn(z.shape, generator=g)
    v, i = t.topk(k, dim=1)
    return v, i.to(torch.int32), torch.logsumexp(t.scatter(1, i, -math.inf) / tau, dim=1) if rest else None


def run_loss(ctx, z, t, tau, labels, alpha, weights, mode, pitch=None, offset=0):
    """mode: step (loss and gradient in one call), onto (the gradient over the logits), later (the gradient by itself)."""
    rows, vocab = z.shape
    dz = R.on_gpu(z, pitch, offset)
    grad = dz if mode == "onto" else R.matrix(rows, vocab, z.dtype, pitch, offset)
    loss, stats = torch.empty(rows, device="cuda"), torch.empty((rows, 4), device="cuda")
    t = [None if x is None else x.cuda() for x in t]
    kw = {"labels": None if labels is None else labels.cuda(), "alpha": alpha}
    w = weights.cuda()
    if mode == "later":
        ctx.he_distill_loss(dz, *t, tau, loss, stats=stats, **kw)
        ctx.he_distill_grad(dz, *t, tau, stats, w, grad, **kw)
    else:
        ctx.he_distill_loss(dz, *t, tau, loss, grad=grad, row_weights=w, **kw)
    around = torch.empty(0, dtype=z.dtype, device="cuda").set_(grad.untyped_storage())
    return loss.cpu().double(), grad.cpu().double(), int(around.isnan().sum()) - (around.numel() - rows * vocab)


def check_loss(got, want, dtype, tau, alpha, weights):
    loss, grad, size = want
    inf = loss.isinf()
    assert torch.equal(got[0][inf], loss[inf])
    d = (got[0] - loss)[~inf].abs()
    assert (d <= 1e-5 * ((1 - alpha) * tau ** 2 + alpha) * (2 + loss[~inf].abs())).all(), float(d.max())
    w = weights.double()[:, None]
    bound = 2e-5 * size * w.abs() + (grad * w).abs() * R.ULP[dtype] * 1.01 + (2.0 ** -25 if dtype == torch.float16 else 1e-38)
    off = (got[1] - grad * w).abs()
    assert (off <= bound).all(), (float((off / bound).max()), divmod(int((off / bound).argmax()), grad.shape[1]))
    assert got[2] == 0


@pytest.mark.parametrize("rows,vocab", [(1, 1), (2, 2), (5, 10), (3, 64), (4, 130), (3, 1000), (2, 1025), (2, 2049), (2, 4097), (2, 9001), (1, 20003), (1, 40000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_loss(ctx, dtype, rows, vocab):
    g = rng(vocab)
    z = (torch.randn((rows, vocab), generator=g) * 3).to(dtype)
    z[0, vocab - vocab // 5:] = -math.inf
    for n, (k, tau, alpha, rest, mode) in enumerate(((1, 1.0, 0.0, False, "step"), (min(vocab, 20), 2.0, 0.1, True, "later"), (min(vocab, 128), 4.0, 0.5, True, "onto"),
                                                     (min(vocab, 33), 1.5, 0.0, True, "step"), (min(vocab, 64), 1.0, 0.3, False, "later"), (2 * vocab if vocab < 64 else 5, 1.0, 1.0, True, "step"))):
        t = teacher(z, min(k, vocab), tau, g, rest)
        if k > vocab:                                        # more entries than indices: the others are not there
            pad = k - vocab
            t = (torch.nn.functional.pad(t[0], (0, pad)), torch.nn.functional.pad(t[1], (0, pad), value=-1), t[2])
        labels = torch.randint(0, max(1, vocab - vocab // 5), (rows,), generator=g, dtype=torch.int32) if alpha else None
        weights = torch.rand(rows, generator=g) + 0.5
        got = run_loss(ctx, z, t, tau, labels, alpha, weights, mode, vocab + n, n)
        check_loss(got, R.distill(z, *t, tau, labels, alpha), dtype, tau, alpha, weights)


@pytest.mark.parametrize("vocab", [40, 1000, 3000])
@pytest.mark.parametrize("mode", ["step", "later", "onto"])
def test_loss_of_rows_that_lack_something(ctx, mode, vocab):
    g, rows, k, tau, alpha = rng(vocab), 14, 16, 2.0, 0.25
    z = torch.randn((rows, vocab), generator=g) * 2
    v, i, r = teacher(z, k, tau, g)
    labels = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    labels[0] = -1                                            # padding
    i[1], r[1] = -1, -math.inf                                # nothing of the teacher
    v[2], r[2] = -math.inf, -math.inf                         # it is -infinity throughout
    i[3, 5:] = -1                                             # fewer entries
    i[4, 2], i[4, 3] = vocab, 2 ** 31 - 1                     # indices that are not there
    z[5] = -math.inf                                          # nothing of the student
    z[6, 10:20] = -math.inf                                   # masked; below, where the teacher has something: the loss is infinite
    z[7, int(i[7, 0])] = -math.inf
    labels[8] = vocab                                         # not there
    labels[9] = int(i[9, 0])                                  # the label is the teacher's first
    i[10, 1] = i[10, 0]                                       # twice
    i[10, 2] = i[10, 0]
    r[11] = -math.inf                                         # no rest
    z[12, int(i[12, 0])] += 150                               # all but sure: what is left is below 2^-100
    z[13] = torch.where(torch.zeros(vocab, dtype=torch.bool).scatter(0, i[13].long(), True), z[13], -math.inf)   # only what is named
    r[13] = -math.inf
    labels[6], labels[7] = (int(i[6, 1]), int(i[7, 1]))
    z[6, int(i[6, 1])], labels[13] = 1.0, int(i[13, 2])
    weights = torch.rand(rows, generator=g) + 0.5
    want = R.distill(z, v, i, r, tau, labels, alpha)
    assert want[0].isinf()[7] and want[0][0] == 0 and want[0][5] == 0
    check_loss(run_loss(ctx, z, (v, i, r), tau, labels, alpha, weights, mode), want, torch.float32, tau, alpha, weights)
    # everything named, nothing left for the rest although the teacher has some: infinite, and no gradient from it
    small, tv, ti = torch.randn((1, 3), generator=g), torch.randn((1, 3), generator=g), torch.tensor([[0, 1, 2]], dtype=torch.int32)
    got = run_loss(ctx, small, (tv, ti, torch.zeros(1)), tau, None, 0.0, torch.ones(1), mode)
    check_loss(got, R.distill(small, tv, ti, torch.zeros(1), tau, None, 0.0), torch.float32, tau, 0.0, torch.ones(1))


def test_gradient_against_differences(ctx):
    """Central differences of the loss itself, h = 2^-4 on logits of size 1: off by h^2/6 of a third derivative (below tau^-1) and by
    the loss's rounding, 1e-5 / h."""
    g, rows, vocab, k, tau, alpha, h = rng(2), 3, 12, 4, 2.0, 0.3, 2.0 ** -4
    z = torch.randn((rows, vocab), generator=g)
    t = teacher(z, k, tau, g)
    labels = torch.tensor([3, int(t[1][1, 0]), 11], dtype=torch.int32)
    _, grad, _ = run_loss(ctx, z, t, tau, labels, alpha, torch.ones(rows), "step")
    for j in range(vocab):
        up, down = z.clone(), z.clone()
        up[:, j] += h
        down[:, j] -= h
        lu, ld = [run_loss(ctx, x, t, tau, labels, alpha, torch.ones(rows), "step")[0] for x in (up, down)]
        assert ((lu - ld) / (2 * h) - grad[:, j]).abs().max() <= h * h / 6 + 1e-3


def test_what_is_not_a_number_stays_in_its_row(ctx):
    g = rng(11)
    z = torch.randn((4, 700), generator=g)
    t = teacher(z, 8, 1.0, g)
    z[1, 300], z[2, 5] = math.nan, math.inf
    loss, grad, _ = run_loss(ctx, z, t, 1.0, None, 0.0, torch.ones(4), "step")
    assert loss[1].isnan() and not loss[2].isfinite() and grad[1].isnan().any() and loss[[0, 3]].isfinite().all() and grad[[0, 3]].isfinite().all()


def test_a_large_vocabulary(ctx):
    g = rng(12)
    z = torch.randn((1, 1 << 20), generator=g) * 2
    t = teacher(z, 100, 2.0, g)
    for mode in ("step", "later", "onto"):
        got = run_loss(ctx, z, t, 2.0, None, 0.0, torch.ones(1), mode)
        check_loss(got, R.distill(z, *t, 2.0, None, 0.0), torch.float32, 2.0, 0.0, torch.ones(1))


@pytest.mark.parametrize("vocab", [1000, 20000])
def test_the_same_call_gives_the_same_bits(ctx, vocab):
    g = rng(13)
    z = (torch.randn((40, vocab), generator=g) * 3).to(torch.bfloat16)
    t = teacher(z, 30, 2.0, g)
    runs = [run_loss(ctx, z, t, 2.0, None, 0.0, torch.ones(40), "step") + run_top(ctx, z, 30, 2.0) for _ in range(3)]
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r[:2] + r[3:], runs[0][:2] + runs[0][3:]))


def test_refusals(ctx):
    from paper_2302_02407_amd.binding import HEError
    z = torch.zeros((4, 100), device="cuda")
    f, i32 = lambda *s: torch.zeros(s, device="cuda"), lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731

    def refused(call, *a, **kw):
        with pytest.raises((HEError, TypeError, ValueError)) as e:
            call(*a, **kw)
        assert not isinstance(e.value, HEError) or e.value.code == -1

    top = ctx.he_top_logits
    refused(top, z, 0.0, f(4, 5), i32(4, 5))
    refused(top, z, math.nan, f(4, 5), i32(4, 5))
    refused(top, z, math.inf, f(4, 5), i32(4, 5))
    refused(top, z, 1.0, f(4, 101), i32(4, 101))                          # more than there are
    refused(top, f(4, 300), 1.0, f(4, 129), i32(4, 129))                  # more than the limit
    refused(top, z, 1.0, f(4, 0), i32(4, 0))
    refused(top, z, 1.0, f(4, 5), i32(4, 6))
    refused(top, z, 1.0, f(4, 5), f(4, 5))
    refused(top, z, 1.0, z[:, :5].contiguous().new_zeros(3, 5), i32(4, 5))
    refused(top, z.double(), 1.0, f(4, 5), i32(4, 5))
    refused(top, z, 1.0, z.view(-1)[:20].view(4, 5), i32(4, 5))           # into the logits
    refused(top, z.expand(4, 100)[:, ::2], 1.0, f(4, 5), i32(4, 5))
    refused(top, z[:1].expand(4, 100), 1.0, f(4, 5), i32(4, 5))           # one row four times: rows overlap
    loss, v, i, r = ctx.he_distill_loss, f(4, 5), i32(4, 5), f(4)
    refused(loss, z, v, i, r, 0.0, f(4))
    refused(loss, z, v, i, r, 1.0, f(4), alpha=0.5)                       # no labels
    refused(loss, z, v, i, r, 1.0, f(4), alpha=1.5, labels=i32(4))
    refused(loss, z, v, i, r, 1.0, f(3))
    refused(loss, z, v, i, r, 1.0, f(4), grad=f(4, 100))                  # no weights
    refused(loss, z, v, i, r, 1.0, f(4), grad=z.bfloat16(), row_weights=f(4))
    refused(loss, z, v, i, r, 1.0, f(4), grad=f(4, 99), row_weights=f(4))
    refused(loss, z, f(4, 129), i32(4, 129), r, 1.0, f(4))
    refused(loss, z, v, i, r, 1.0, r)                                     # onto the teacher's
    room = f(5, 100)
    refused(loss, room[:4], v, i, r, 1.0, f(4), grad=room[1:], row_weights=f(4))
    refused(ctx.he_distill_grad, z, v, i, r, 1.0, f(4, 3), f(4), f(4, 100))
    refused(ctx.he_distill_grad, z, v, i, r, 1.0, f(4, 4), None, f(4, 100))
    top(z[:0], 1.0, f(0, 5), i32(0, 5))                                   # no rows: fine
    loss(z[:0], v[:0], i[:0], None, 1.0, f(0))
    torch.cuda.synchronize()


def with_masks(rows, vocab, low, seed):
    """Rows with some logits, all but two, all, and none at the lowest value."""
    z = 3 * torch.randn((rows, vocab), generator=rng(seed))
    z[0::4][torch.rand((len(z[0::4]), vocab), generator=rng(seed + 1)) < 0.7] = low
    z[1::4] = torch.where((torch.arange(vocab) == 1) | (torch.arange(vocab) == vocab - 1), z[1::4], low)
    z[2::4] = low
    return z


LOWS = [(torch.float32, torch.finfo(torch.float32).min), (torch.float32, -1e38), (torch.bfloat16, torch.finfo(torch.bfloat16).min), (torch.bfloat16, -3.0e38)]


@pytest.mark.parametrize("vocab", [3, 10, 700, 9001, 40000])
@pytest.mark.parametrize("tau", [0.25, 1.0, 3.0])
@pytest.mark.parametrize("dtype,low", LOWS)
def test_top_of_rows_masked_by_the_lowest_value(ctx, vocab, tau, dtype, low):
    z = with_masks(8, vocab, low, vocab).to(dtype)
    k = min(5, vocab)
    got, (values, index, _) = run_top(ctx, z, k, tau), R.top(z, k, tau)
    check_top(got, (values, index, R.top(torch.where(z.double() <= -1e37, -math.inf, z.double()), k, tau)[2]))
    assert (got[2][2::4] == -math.inf).all()


@pytest.mark.parametrize("tau", [0.5, 1.0])
def test_top_of_numbers_that_overflow_a_sum(ctx, tau):
    z = torch.randn((3, 5000), generator=rng(0))
    z[0, 17], z[0, 4000] = 3.3e38, 3.2e38
    z[1, 9], z[1, 11] = 3.3e38, -3.3e38
    got, want = run_top(ctx, z, 1, tau), R.top(z, 1, tau)
    assert torch.equal(got[1], want[1]) and got[2][0] == math.inf
    check_top([g[1:] for g in got], [w[1:] for w in want])


@pytest.mark.parametrize("vocab", [3, 10, 700, 9001, 40000])
@pytest.mark.parametrize("tau", [0.25, 1.0, 3.0])
@pytest.mark.parametrize("with_rest", [False, True])
@pytest.mark.parametrize("dtype,low", LOWS)
@pytest.mark.parametrize("mode", ["step", "later"])
def test_distillation_of_rows_masked_by_the_lowest_value(ctx, vocab, tau, with_rest, dtype, low, mode):
    """As if the masked logits were -infinity.  The teacher's indices and the label are among those that are not masked; what it names of a row that is
    masked throughout does not matter."""
    rows, k = 8, min(4, vocab)
    z = with_masks(rows, vocab, low, vocab + 1).to(dtype)
    as_meant = torch.where(z.double() <= -1e37, -math.inf, z.double())
    order = as_meant.argsort(dim=1, descending=True, stable=True)
    index = torch.where(as_meant.gather(1, order[:, :k]) > -math.inf, order[:, :k], -1).to(torch.int32)
    values = 2 * torch.randn((rows, k), generator=rng(1))
    rest = torch.randn(rows, generator=rng(2)) if with_rest else None
    if with_rest:                                             # where nothing else is left, the teacher has nothing else either
        rest = torch.where((as_meant > -math.inf).sum(dim=1) > (index >= 0).sum(dim=1), rest, -math.inf)
    labels, weights = order[:, 0].to(torch.int32), torch.rand(rows, generator=rng(3)) + 0.5
    want = R.distill(as_meant, values, index, rest, tau, labels, 0.25)
    got = run_loss(ctx, z, (values, index, rest), tau, labels, 0.25, weights, mode, vocab + 1, 1)
    check_loss(got, want, dtype, tau, 0.25, weights)
    assert (got[0][2::4] == 0).all() and (got[1][2::4] == 0).all()


@pytest.mark.parametrize("vocab,k", [(300, 7), (1000, 20), (1024, 100), (513, 1)])
@pytest.mark.parametrize("mode", ["step", "later", "onto"])
def test_loss_of_many_short_rows(ctx, vocab, k, mode):
    """From 1024 rows on one wavefront takes a row of up to 4 KB."""
    rows, tau, g = 1030, 2.0, rng(vocab)
    dtype = torch.float32 if vocab != 513 else torch.bfloat16
    z, t = (2 * torch.randn((rows, vocab), generator=g)).to(dtype), 2 * torch.randn((rows, vocab), generator=g)
    values, index, rest = R.top(t, k, tau)
    values, index, rest = values.float(), index.to(torch.int32), rest.float()
    labels = torch.randint(-1, vocab + 1, (rows,), generator=g, dtype=torch.int32)
    weights = torch.rand(rows, generator=g) + 0.5
    want = R.distill(z, values, index, rest, tau, labels, 0.25)
    check_loss(run_loss(ctx, z, (values, index, rest), tau, labels, 0.25, weights, mode, vocab + 3, 1), want, dtype, tau, 0.25, weights)


@pytest.mark.parametrize("vocab,k", [(40, 40), (120, 120), (200, 32), (256, 33), (511, 1), (512, 32)])
@pytest.mark.parametrize("dtype", TYPES)
def test_top_of_short_rows(ctx, vocab, k, dtype):
    """In order, all equal, with NaN, masked and in no order: rows that one wavefront takes, and such as it leaves to four."""
    g = rng(vocab + k)
    z = torch.randn((8, vocab), generator=g).to(dtype)
    z[1] = z[1].sort().values
    z[2] = z[2].sort(descending=True).values
    z[3] = 0.5
    z[4, ::3] = -math.inf
    z[5] = -math.inf
    z[6, vocab // 2], z[6, 1] = math.nan, math.inf
    z[7, : vocab // 2] = z[7, 0]
    check_top(run_top(ctx, z, k, 1.5, vocab + 1, 1), R.top(z, k, 1.5))
