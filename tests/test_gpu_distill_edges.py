"""GPU: the distillation loss and its gradient, and the top logits, at the edges of what their definitions say.

Tolerances are those of the ordinary rows (test_gpu_distill.py): an edge changes what a row's result is, not how it is rounded."""
import itertools
import math

import pytest
import torch

import plain_ref as R
from test_gpu_distill import check_loss, check_top, rng, run_loss, run_top, teacher, with_masks

pytestmark = pytest.mark.gpu
MODES = ["step", "later", "onto"]


@pytest.fixture(scope="module")
def ctx():
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    return HEContext.from_params(config_params(0))


def rows_of(result, rows):
    """Some rows of (loss, gradient, ...)."""
    return tuple(x[rows] for x in result[:2]) + tuple(result[2:])


@pytest.mark.parametrize("vocab", [3, 10, 700, 9001, 40000])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_label_of_a_gradient_taken_later(ctx, vocab, tau):
    """One lane reads the label's logit, all of its wavefront use it; the gradient alone takes no sum in between."""
    g, rows, alpha = rng(vocab), 33, 0.5
    z = 3 * torch.randn((rows, vocab), generator=g)
    t = teacher(z, min(vocab, 2), tau, g)
    labels = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    weights = torch.rand(rows, generator=g) + 0.5
    want = R.distill(z, *t, tau, labels, alpha)
    check_loss(run_loss(ctx, z, t, tau, labels, alpha, weights, "later"), want, torch.float32, tau, alpha, weights)


def by_definition(z, values, index, rest, tau, labels, alpha):
    """(loss, gradient, the sum of what its terms amount to) for distinct entries that are all there.  The rest's share of each logit is a softmax of its
    own: from logarithms of probabilities, as far below 0 as logits can be, it would be lost to rounding in 64 bits."""
    x, at = z.double(), index.long()
    t = torch.cat([values.double() / tau, torch.full((len(z), 1), -math.inf).double() if rest is None else rest.double()[:, None]], dim=1)
    p, logp = torch.softmax(t, dim=1), torch.log_softmax(t, dim=1)
    named = torch.zeros(z.shape, dtype=torch.bool).scatter_(1, at, True)
    logq, others = torch.log_softmax(x / tau, dim=1), torch.where(named, -math.inf, x / tau)
    kl, parts = (p[:, :-1] * (logp[:, :-1] - logq.gather(1, at))).sum(dim=1), [torch.softmax(x / tau, dim=1), -torch.zeros_like(x).scatter_(1, at, p[:, :-1])]
    if rest is not None:
        kl += p[:, -1] * (logp[:, -1] - torch.logsumexp(torch.where(named, -math.inf, logq), dim=1))
        parts.append(-p[:, -1:] * torch.softmax(others, dim=1))
    loss, parts = (1 - alpha) * tau ** 2 * kl, [(1 - alpha) * tau * q for q in parts]
    if labels is not None:
        y = labels.long()[:, None]
        loss -= alpha * torch.log_softmax(x, dim=1).gather(1, y)[:, 0]
        parts += [alpha * torch.softmax(x, dim=1), -alpha * torch.zeros_like(x).scatter_(1, y, 1.0)]
    return loss, sum(parts), sum(q.abs() for q in parts)


FAR = [-1e9, -1e10, -3e12, -1e20, -1e30, -1e36]


@pytest.mark.parametrize("vocab", [3, 10, 700, 9001, 40000])
@pytest.mark.parametrize("mode", ["step", "later"])
def test_distillation_with_masks_that_are_numbers(ctx, mode, vocab):
    """Masks of -1e9 to -1e36 are logits like others: beside real ones they are nothing, and a row of nothing else is uniform."""
    g, alpha = rng(vocab), 0.25
    for low, dtype, (tau, with_rest) in itertools.product(FAR, (torch.float32, torch.bfloat16), ((0.25, True), (1.0, False), (1.0, True), (3.0, False), (3.0, True))):
        z = with_masks(8, vocab, low, vocab + 1).to(dtype)
        t = teacher(torch.randn((8, vocab), generator=g), min(vocab - 1, 4), tau, g, with_rest)
        labels, weights = z.double().argmax(dim=1).to(torch.int32), torch.rand(8, generator=g) + 0.5
        want = by_definition(z, *t, tau, labels, alpha)
        check_loss(run_loss(ctx, z, t, tau, labels, alpha, weights, mode, vocab + 1, 1), want, dtype, tau, alpha, weights)


@pytest.mark.parametrize("vocab", [3, 40, 700, 9001, 40000])
@pytest.mark.parametrize("tau,alpha,with_rest", [(0.25, 0.0, True), (1.0, 0.0, False), (1.0, 0.5, True), (4.0, 0.5, True), (4.0, 0.5, False)])
def test_distillation_of_large_logits(ctx, tau, alpha, with_rest, vocab):
    """Logits around a number of any size: what counts is how they differ.  Losses that 32 bits do not hold are infinite."""
    g, rows = rng(vocab), 8
    z = 3 * torch.randn((rows, vocab), generator=g)
    t = teacher(z, 2, tau, g, with_rest)
    z += torch.tensor([1e4, -1e6, 1e8, -1e8, 1e10, 1e20, 1e30, -1e30])[:, None]
    z[5, int(t[1][5, 0])] = 3e20
    z[6, vocab // 2] = 3.2e38
    labels, weights = t[1][:, 0].clone() if alpha else None, torch.rand(rows, generator=g) + 0.5
    loss, grad, size = by_definition(z, *t, tau, labels, alpha)
    loss = torch.where(loss > 3.4e38, math.inf, loss)
    for mode in ("step", "later"):
        check_loss(run_loss(ctx, z, t, tau, labels, alpha, weights, mode), (loss, grad, size), torch.float32, tau, alpha, weights)


@pytest.mark.parametrize("vocab", [3, 10, 200, 700, 1000, 9001, 40000])
def test_top_with_masks_that_are_numbers(ctx, vocab):
    for low, dtype, tau in itertools.product(FAR, (torch.float32, torch.bfloat16), (0.25, 1.0, 3.0)):
        z = with_masks(8, vocab, low, vocab).to(dtype)
        for k in (1, min(5, vocab)):
            check_top(run_top(ctx, z, k, tau, vocab + 1, 1), R.top(z, k, tau))


@pytest.mark.parametrize("vocab", [3, 40, 700, 9001, 40000])
def test_top_of_large_logits(ctx, vocab):
    z = 3 * torch.randn((8, vocab), generator=rng(vocab))
    z += torch.tensor([1e4, -1e6, 1e8, -1e8, 1e10, 1e20, 1e30, -1e30])[:, None]
    z[5, vocab // 2], z[6, vocab // 3] = 3e20, 1e36
    for k, tau in itertools.product((1, min(20, vocab)), (0.25, 1.0, 30.0)):
        check_top(run_top(ctx, z, k, tau), R.top(z, k, tau))


def spoilt_teacher(z, tau, g, with_rest):
    """A teacher that is not finite in rows 1, 3, 5 and 6 (the last two in what it gives the rest), and in an entry of row 7 that is not there."""
    v, i, r = teacher(z, 3, tau, g, with_rest)
    v[1, 2], v[3, 0], v[7, 1], i[7, 1] = math.nan, math.inf, math.nan, -1
    if with_rest:
        r[5], r[6] = math.nan, math.inf
    return (v, i, r), [1, 3, 5, 6] if with_rest else [1, 3]


@pytest.mark.parametrize("vocab", [3, 40, 700, 9001, 40000])
@pytest.mark.parametrize("with_rest", [False, True])
@pytest.mark.parametrize("mode", MODES)
def test_a_teacher_that_is_not_finite(ctx, mode, with_rest, vocab):
    """Its distribution is not one of numbers, and neither is the loss: never a finite one without a sign of it."""
    g, rows, tau, alpha = rng(vocab), 9, 2.0, 0.25
    z = 2 * torch.randn((rows, vocab), generator=g)
    t, spoilt = spoilt_teacher(z, tau, g, with_rest and vocab > 3)
    labels = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    weights = torch.rand(rows, generator=g) + 0.5
    got = run_loss(ctx, z, t, tau, labels, alpha, weights, mode, vocab + 1, 1)
    loss, grad = got[:2]
    assert loss[spoilt].isnan().all() and grad[spoilt].isnan().any(dim=1).all()
    sound = [r for r in range(rows) if r not in spoilt]
    want = R.distill(z, t[0].nan_to_num(nan=0.0), *t[1:], tau, labels, alpha)          # row 7's entry is not there
    check_loss(rows_of(got[:2], sound) + (0,), rows_of(want[:2], sound) + (want[2][sound],), torch.float32, tau, alpha, weights[sound])


@pytest.mark.parametrize("vocab", [3, 40, 700, 9001, 40000])
@pytest.mark.parametrize("mode", MODES)
def test_a_term_that_is_not_there_adds_nothing(ctx, mode, vocab):
    """With alpha = 1 the teacher does not count, whatever it is; a row that has neither term has no gradient, whatever the student is."""
    g, rows, tau = rng(vocab), 9, 2.0
    z = 2 * torch.randn((rows, vocab), generator=g)
    t, _ = spoilt_teacher(z, tau, g, vocab > 3)
    labels = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    weights = torch.rand(rows, generator=g) + 0.5
    any_finite = [None if x is None else x.nan_to_num(nan=0.0, posinf=0.0) for x in t]
    check_loss(run_loss(ctx, z, t, tau, labels, 1.0, weights, mode), R.distill(z, *any_finite, tau, labels, 1.0), torch.float32, tau, 1.0, weights)
    none = [torch.zeros((rows, 3)), torch.full((rows, 3), -1, dtype=torch.int32), None]
    z[1, vocab // 2], z[3, 0], z[4], z[5] = math.nan, math.inf, math.nan, -math.inf
    labels[:] = vocab
    loss, grad, _ = run_loss(ctx, z, none, tau, None, 0.0, weights, mode)
    assert (loss == 0).all() and (grad == 0).all()
    for alpha in (0.25, 1.0):
        loss, grad, _ = run_loss(ctx, z, none, tau, labels, alpha, weights, mode)
        assert (loss == 0).all() and (grad == 0).all()
    labels[:] = 0
    loss, grad, _ = run_loss(ctx, z, none, tau, labels, 0.25, weights, mode)       # one of the two is there
    assert loss[[1, 3, 4]].isnan().all() and grad[[1, 3, 4]].isnan().any(dim=1).all() and grad[[0, 2, 5, 6, 7, 8]].isfinite().all()


def test_temperatures_that_32_bits_do_not_carry(ctx):
    """From 2^-60 to 2^60 a row's factors (log2(e) / tau, tau^2) and a masked logit's power are what they should be; others are refused."""
    from paper_2302_02407_amd.binding import HEError
    g = rng(1)
    z = torch.randn((5, 700), generator=g)
    z[1:3, 100:600] = torch.finfo(torch.float32).min
    z[3] = torch.finfo(torch.float32).min
    for tau in (2.0 ** -60, 2.0 ** 60):
        got, (values, index, _) = run_top(ctx, z, 5, tau), R.top(z, 5, tau)
        check_top(got, (values, index, R.top(torch.where(z < -1e30, -math.inf, z.double()), 5, tau)[2]))
    d, v, i, r = z.cuda(), torch.zeros((5, 4), device="cuda"), torch.zeros((5, 4), dtype=torch.int32, device="cuda"), torch.zeros(5, device="cuda")
    for tau in (2.0 ** -61, 2.0 ** 61, 1e-40, 1e38):
        for call in (lambda: ctx.he_top_logits(d, tau, v, i, r), lambda: ctx.he_distill_loss(d, v, i, r, tau, torch.zeros(5, device="cuda")),
                     lambda: ctx.he_distill_grad(d, v, i, r, tau, torch.zeros((5, 4), device="cuda"), r, torch.zeros_like(d))):
            with pytest.raises(HEError) as e:
                call()
            assert e.value.code == -1
    for tau in (2.0 ** -60, 2.0 ** 60):
        ctx.he_distill_loss(d, v, i, None, tau, r)
    torch.cuda.synchronize()
