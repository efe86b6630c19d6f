"""GPU: what the plaintext side's sequencing chooses for a caller, and takes from one."""

import pytest
import torch

import plain_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    return HEContext.from_params(config_params(0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_a_heads_sums_are_exact_unless_results_have_16_bits(ctx, dtype):
    """Logits of 32 bits lose nothing that the caller did not give away."""
    from paper_2302_02407_amd.distill import TeacherHead
    rows, vocab, dim = 150, 700, 512                          # tiles that have both kinds of sums
    g = torch.Generator().manual_seed(1)
    table, x = (torch.randn((vocab, dim), generator=g) / 20).cuda(), torch.randn((rows, dim), generator=g).cuda()
    logits = {}
    for fast in (None, False, True):
        head = TeacherHead(ctx, table, None, rows, 4, 1.0, dtype=dtype) if fast is None else TeacherHead(ctx, table, None, rows, 4, 1.0, dtype=dtype, fast_sums=fast)
        head(x)
        logits[fast] = head.logits.clone()
    assert torch.equal(logits[None], logits[dtype != torch.float32])
    assert not torch.equal(logits[False], logits[True]) or dtype != torch.float32


def test_labels_of_64_bits(ctx):
    """Labels as losses of torch take them; one that 32 bits do not hold is padding or not there, as its sign says."""
    from paper_2302_02407_amd.distill import Answers, distill_loss
    g, rows, vocab = torch.Generator().manual_seed(2), 40, 300
    z = torch.randn((rows, vocab), generator=g)
    values, index, rest = R.top(z + torch.randn((rows, vocab), generator=g), 5, 2.0)
    answers = Answers(values.float().cuda(), index.to(torch.int32).cuda(), rest.float().cuda())
    labels = torch.randint(0, vocab, (rows,), generator=g)
    labels[:6] = torch.tensor([-100, 2 ** 40, -2 ** 40, 2 ** 32 + 3, -2 ** 32 + 3, vocab])
    small = labels.clamp(-1, vocab).to(torch.int32)
    grads, losses = [], []
    for y in (labels, small):
        d = z.cuda().requires_grad_()
        loss = distill_loss(ctx, d, answers, 2.0, y.cuda(), 0.3)
        loss.sum().backward()
        losses.append(loss.detach())
        grads.append(d.grad)
    assert torch.equal(*losses) and torch.equal(*grads)
    assert (losses[0][[0, 2, 4]] == 0).all() and (losses[0][[1, 3, 5]] != 0).all()


def test_one_row_of_any_pitch(ctx):
    """How far a single row's next one would be does not matter."""
    g = torch.Generator().manual_seed(3)
    dim, n = 96, 40
    x = torch.randn((3, 101), generator=g).cuda()[:1, :dim]
    codes, scales = torch.zeros((3, 100), dtype=R.F8, device="cuda")[:1, :dim], torch.zeros((3, 7), device="cuda")[:1, :1]
    ctx.he_rmsnorm_q8(x, codes, scales, 1e-6)
    near = torch.zeros((1, dim), dtype=R.F8, device="cuda"), torch.zeros((1, 1), device="cuda")
    ctx.he_rmsnorm_q8(x.contiguous(), *near, 1e-6)
    assert torch.equal(codes.view(torch.uint8), near[0].view(torch.uint8)) and torch.equal(scales, near[1])
    w, sw, out, want = torch.randn((n, dim), generator=g).to(R.F8).cuda(), torch.ones((1, 1), device="cuda"), torch.zeros((1, n), device="cuda"), torch.zeros((1, n), device="cuda")
    ctx.he_matmul_q8(codes, scales, w, sw, out)
    ctx.he_matmul_q8(*near, w, sw, want)
    assert torch.equal(out, want)
    one = w.as_strided((1, dim), (1 << 29, 1))                # a pitch that rows could not have
    ctx.he_matmul_q8(codes, scales, one, sw, out[:, :1])
    assert torch.equal(out[:, :1], want[:, :1])
    z = torch.randn((2, 700), generator=g).cuda()
    values, index = torch.zeros((1, 3), device="cuda"), torch.zeros((1, 3), dtype=torch.int32, device="cuda")
    ctx.he_top_logits(z.as_strided((1, 700), (1 << 29, 1)), 1.0, values, index)
    assert torch.equal(index.cpu().long(), R.top(z[:1].cpu(), 3, 1.0)[1])


def test_logits_that_are_not_rows_of_their_own(ctx):
    """One student's row against several answers, and columns of a larger matrix: the gradient goes where the logits come from."""
    from paper_2302_02407_amd.distill import Answers, distill_loss
    g, rows, vocab, tau = torch.Generator().manual_seed(4), 7, 120, 2.0
    values, index, rest = R.top(torch.randn((rows, vocab), generator=g), 5, tau)
    answers = Answers(values.float().cuda(), index.to(torch.int32).cuda(), rest.float().cuda())
    for shape, view in (((vocab,), lambda t: t.expand(rows, vocab)), ((1, vocab), lambda t: t.expand(rows, vocab)), ((rows, 2 * vocab), lambda t: t[:, ::2]),
                        ((vocab, rows), lambda t: t.T), ((rows, vocab + 3), lambda t: t[:, 3:]), ((rows * vocab // 2 + vocab,), lambda t: t.as_strided((rows, vocab), (vocab // 2, 1)))):
        z = torch.randn(shape, generator=g)
        want, dz, size = R.distill(view(z), *(t.cpu() for t in answers), tau, None, 0.0)
        ref = z.double().requires_grad_()
        view(ref).backward(dz)
        most = z.double().requires_grad_()
        view(most).backward(size)
        d = z.cuda().requires_grad_()
        loss = distill_loss(ctx, view(d), answers, tau)
        loss.sum().backward()
        assert ((loss.detach().cpu().double() - want).abs() <= 1e-5 * tau ** 2 * (2 + want.abs())).all()
        assert ((d.grad.cpu().double() - ref.grad).abs() <= 2e-5 * most.grad + 1e-38).all()
