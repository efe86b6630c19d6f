"""GPU: what the plaintext side's sequencing chooses for a caller, and takes from one."""
import math

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
