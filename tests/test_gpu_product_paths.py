"""GPU: the product of 8-bit codes on each of its ways through a long sum: every block of 128 columns with scales of its own.

Codes are whole numbers up to 8, so that a block's sum is exact either way (a fast sum drops of a product what is 2^-13 of its group's largest, at most
64).  What remains are a block's product with its scales and its addition, in the reference too: 2^-24 of the terms' magnitudes each."""
import pytest
import torch

import plain_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    return HEContext.from_params(config_params(0))


WAYS = [(3, 16400, 300), (16, 16390, 1300), (2, 98500, 600),           # few rows, two tiles of W a wavefront: one block each, and two
        (24, 1010, 9000),                                              # ... up to 32 rows, five blocks a wavefront
        (1, 32768, 1100), (20, 16500, 2100), (30, 2050, 20000),        # tiles of 32 rows, in parts of 5, 5 and 10 blocks
        (50, 66000, 1100), (50, 2300, 20000),                          # of 64: 9 blocks at once; parts of 10
        (777, 10007, 2040), (1100, 8000, 2100), (200, 2500, 20470),    # of 128: 16 and 17 blocks at once, the last a partial one; parts of 13
        (3590, 4090, 2100), (3600, 4100, 1024)]                        # of 256: 17 blocks, and eight, the scales' whole first fill


@pytest.mark.parametrize("m,n,k", WAYS)
def test_scales_of_every_block(ctx, m, n, k):
    g = torch.Generator().manual_seed(n)
    a, w = [torch.randint(-8, 9, (r, k), generator=g).float() for r in (m, n)]
    kb = -(-k // 128)
    sa, sw = torch.rand((m, kb), generator=g) + 0.01, torch.rand((-(-n // 128), kb), generator=g) + 0.01
    want, size = torch.zeros((m, n)), torch.zeros((m, n))
    for b in range(kb):
        at = slice(128 * b, 128 * b + 128)
        part = (a[:, at] @ w[:, at].T) * sa[:, b:b + 1] * sw[:, b].repeat_interleave(128)[:n]
        want += part
        size += part.abs()
    da, dw, dsa, dsw = R.code_rows(a.to(R.F8)), R.code_rows(w.to(R.F8)), sa.cuda(), sw.cuda()
    for dtype, fast in ((torch.float32, False), (torch.bfloat16, True), (torch.float16, True), (torch.bfloat16, False)):
        out = R.matrix(m, n, dtype, n + 3, 1)
        ctx.he_matmul_q8(da, dsa, dw, dsw, out, fast_sums=fast)
        off = (out.cpu().float() - want).abs()
        bound = size * ((kb + 4) * 2.0 ** -23) + want.abs() * R.ULP[dtype] * 1.01 + (2.0 ** -25 if dtype == torch.float16 else 0)
        assert (off <= bound).all(), (dtype, fast, float((off / bound.clamp_min(1e-30)).max()))
        assert int(torch.empty(0, dtype=dtype, device="cuda").set_(out.untyped_storage()).isnan().sum()) == out.untyped_storage().nbytes() // out.element_size() - m * n
