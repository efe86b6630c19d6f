"""GPU: the norm with 8-bit output on rows whose squares leave the range of 32 bits, and without a term under the root to hold it off zero."""
import pytest
import torch

import plain_ref as R
from test_gpu_q8_head import check_norm, rng

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    return HEContext.from_params(config_params(0))


def run(ctx, x, r, w, eps, sound=slice(None)):
    """Codes and scales; those of the rows `sound`, which have a root to be divided by, are what the definition says."""
    rows, dim = x.shape
    codes, scales = R.code_rows(torch.zeros((rows, dim), dtype=R.F8)), R.matrix(rows, -(-dim // 128), torch.float32)
    total = R.matrix(rows, dim, x.dtype) if r is not None else None
    ctx.he_rmsnorm_q8(x.cuda(), codes, scales, eps, residual=None if r is None else r.cuda(), weight=None if w is None else w.cuda(), sum_out=total)
    check_norm(x[sound], None if r is None else r[sound], w, eps, codes[sound], scales[sound], None if r is None else total[sound], x.dtype)
    return codes.cpu().float(), scales.cpu()


@pytest.mark.parametrize("dim", [5, 128, 300, 1001, 1700, 5000, 9000, 20000, 40000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_zeros_without_eps(ctx, dtype, dim):
    """A block of zeros has scale 0 and codes 0, in a row of nothing else too."""
    g = rng(dim)
    x = torch.randn((6, dim), generator=g).to(dtype)
    x[1], x[4], x[2, :dim // 2] = 0, -0.0, 0
    w = (1 + 0.1 * torch.randn(dim, generator=g)).to(dtype)
    for weight in (None, w):
        codes, scales = run(ctx, x, None, weight, 0.0, [0, 2, 3, 5])
        assert (scales[[1, 4]] == 0).all() and (codes[[1, 4]] == 0).all()
    r = torch.randn((6, dim), generator=g).to(dtype)
    r[1], r[2, :dim // 2], r[4] = 0, 0, 0
    codes, scales = run(ctx, x, r, w, 0.0, [0, 2, 3, 5])
    assert (scales[[1, 4]] == 0).all() and (codes[[1, 4]] == 0).all()


@pytest.mark.parametrize("dim", [5, 300, 1001, 1700, 5000, 9000, 20000, 40000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -133, 1e-6, 2.0 ** 90])
def test_squares_beyond_the_range(ctx, eps, dtype, dim):
    """Rows from the smallest numbers to the largest: y = h / sqrt(mean(h^2) + eps) is of size 1 although h^2 is not a number of 32 bits."""
    g, sizes = rng(dim), [2.0 ** -131, 1e-36, 1e-30, 1e-22, 1e-18, 1.0, 1e18, 2e19, 1e25, 1e37]
    eps = float(torch.tensor(eps))
    x = torch.randn((len(sizes), dim), generator=g).clamp_(-4, 4) * torch.tensor(sizes)[:, None]
    x[-1, dim // 2] = 3e38
    x, w = x.to(dtype), (1 + 0.1 * torch.randn(dim, generator=g)).to(dtype)
    run(ctx, x, None, None, eps)
    run(ctx, x, None, w, eps)
    r = (0.25 * x.float()).flip(1).to(dtype)
    r[-1] = 0
    run(ctx, x, r, w, eps)
