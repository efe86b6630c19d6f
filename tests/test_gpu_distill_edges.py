"""GPU: the distillation loss and its gradient, and the top logits, at the edges of what their definitions say.

Tolerances are those of the ordinary rows (test_gpu_distill.py): an edge changes what a row's result is, not how it is rounded."""
import math

import pytest
import torch

import plain_ref as R
from test_gpu_distill import check_loss, check_top, rng, run_loss, run_top, teacher

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
