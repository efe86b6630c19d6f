"""GPU: the plaintext operators on rows so far apart that offsets pass 32 bits, in a captured graph, and on nothing at all."""
import pytest
import torch

import plain_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    return HEContext.from_params(config_params(0))


def far(t, pitch):
    """t's rows on the GPU, `pitch` elements apart; what lies between is whatever was there."""
    rows, cols = t.shape
    m = torch.empty((rows - 1) * pitch + -(-cols // 16) * 16, dtype=t.dtype, device="cuda")[:(rows - 1) * pitch + cols].as_strided((rows, cols), (pitch, 1))
    return m.copy_(t.cuda())


@pytest.mark.parametrize("step", [True, False])
def test_far_logits(ctx, step):
    rows, vocab, k, pitch = 18, 1000, 8, 1 << 28                  # 17 * 2^28 elements: past 2^32
    g = torch.Generator().manual_seed(1)
    z = torch.randn((rows, vocab), generator=g).to(torch.bfloat16)
    d = far(z, pitch)
    v, i, r = torch.empty((rows, k), device="cuda"), torch.empty((rows, k), dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    ctx.he_top_logits(d, 1.5, v, i, r)
    values, index, rest = R.top(z, k, 1.5)
    assert torch.equal(i.cpu().long(), index) and torch.equal(v.cpu().double(), values) and ((r.cpu().double() - rest).abs() <= 1e-5 * (1 + rest.abs())).all()
    student = torch.randn((rows, vocab), generator=g).to(torch.bfloat16)
    want, dz, size = R.distill(student, v.cpu(), i.cpu(), r.cpu(), 1.5, None, 0.0)
    d.copy_(student.cuda())
    near, weights = student.cuda(), torch.ones(rows, device="cuda")
    for a, b in ((d, torch.empty_like(near)), (near, d)):         # far logits, then a far gradient over them
        loss, stats = torch.empty(rows, device="cuda"), torch.empty((rows, 4), device="cuda")
        if step:
            ctx.he_distill_loss(a, v, i, r, 1.5, loss, grad=b, row_weights=weights)
        else:
            ctx.he_distill_loss(a, v, i, r, 1.5, loss, stats=stats)
            ctx.he_distill_grad(a, v, i, r, 1.5, stats, weights, b)
        assert ((loss.cpu().double() - want).abs() <= 1e-5 * 1.5 ** 2 * (2 + want.abs())).all()
        assert ((b.cpu().double() - dz).abs() <= 2e-5 * size + dz.abs() * R.ULP[torch.bfloat16] * 1.01 + 1e-38).all()


def test_far_rows_of_the_head(ctx):
    """Whole numbers, so that every sum is exact, as the codes of a norm's rows are when told from its scales."""
    m, n, k, pitch = 600, 530, 144, 1 << 23                       # 600 * 2^23 codes: past 2^32
    g = torch.Generator().manual_seed(2)
    a, w = [torch.randint(-8, 9, (r, k), generator=g).float() for r in (m, n)]
    ones = [torch.ones((r, 2), device="cuda") for r in (m, -(-n // 128))]
    for rows in (m, 3):                                           # tiles; and the kernel for few rows
        da, dw, out = far(a[:rows].to(R.F8), pitch), far(w.to(R.F8), pitch), far(torch.zeros((rows, n)), pitch)
        for fast in (False, True):
            ctx.he_matmul_q8(da, ones[0][:rows], dw, ones[1], out, fast_sums=fast)
            assert torch.equal(out.cpu(), a[:rows] @ w.T)
    del da, dw, out
    x = torch.randn((18, 200), generator=g)
    near_codes, near_scales = R.code_rows(torch.zeros((18, 200), dtype=R.F8)), torch.empty((18, 2), device="cuda")
    ctx.he_rmsnorm_q8(x.cuda(), near_codes, near_scales, 1e-6)
    far_codes, far_scales = far(torch.zeros((18, 200), dtype=R.F8), 1 << 28), far(torch.zeros((18, 2)), 1 << 28)
    ctx.he_rmsnorm_q8(far(x, 1 << 28), far_codes, far_scales, 1e-6)
    assert torch.equal(far_codes.cpu().view(torch.uint8), near_codes.cpu().view(torch.uint8)) and torch.equal(far_scales.cpu(), near_scales.cpu())


def test_in_a_graph():
    """The whole path captured once and replayed on other inputs, with eager work between the replays."""
    from he_inputs.params import config_params
    from paper_2302_02407_amd.binding import HEContext
    from paper_2302_02407_amd.distill import TeacherHead
    rows, vocab, dim, k = 96, 600, 2048, 16                       # a product in parts: its workspace is reserved before
    g = torch.Generator().manual_seed(4)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = HEContext.from_params(config_params(0))
        ctx.he_ws_reserve(max(1, ctx.he_ws_query_matmul_q8(rows, vocab, dim)))
        head = TeacherHead(ctx, torch.randn((vocab, dim), generator=g).cuda() / 32, None, rows, k, 2.0)
        x, z = torch.zeros((rows, dim), device="cuda"), torch.zeros((rows, vocab), device="cuda")
        loss, grad, weights = torch.empty(rows, device="cuda"), torch.empty((rows, vocab), device="cuda"), torch.ones(rows, device="cuda")

        def run():
            answers = head(x)
            ctx.he_distill_loss(z, *answers, 2.0, loss, grad=grad, row_weights=weights)
            return answers

        run()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            captured = run()
        for seed in range(4):
            x.copy_(torch.randn((rows, dim), generator=g))
            z.copy_(torch.randn((rows, vocab), generator=g))
            graph.replay()
            stream.synchronize()
            got = [t.clone() for t in (*captured, loss, grad)]
            answers = run()
            stream.synchronize()
            for a, b in zip(got, (*answers, loss, grad)):
                assert torch.equal(a, b)


def test_no_rows(ctx):
    from paper_2302_02407_amd.distill import TeacherHead
    head = TeacherHead(ctx, torch.ones((40, 64), device="cuda"), None, 4, 3, 1.0)
    answers = head(torch.zeros((0, 64), device="cuda"))
    assert [t.shape[0] for t in answers] == [0, 0, 0]
    ctx.he_distill_loss(torch.zeros((0, 40), device="cuda"), *answers, 1.0, torch.zeros(0, device="cuda"))
    ctx.he_matmul_q8(torch.zeros((0, 64), dtype=R.F8, device="cuda"), torch.zeros((0, 1), device="cuda"), torch.zeros((8, 64), dtype=R.F8, device="cuda"),
                     torch.zeros((1, 1), device="cuda"), torch.zeros((0, 8), device="cuda"))
