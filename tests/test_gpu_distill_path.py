"""From a teacher's last hidden state to a student that runs on ciphertexts: the plaintext operators as they are used together."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

import plain_ref as R
from he_inputs import sampling as S
from he_inputs.params import toy_params

pytestmark = pytest.mark.gpu


def small_ring():
    return toy_params(logN=10, q_bits=40, nq=3, p_bits=41, np_=1, dnum=3, scale=2.0 ** 30, hamming=32, seed=80)


@pytest.fixture(scope="module")
def ctx():
    from paper_2302_02407_amd.binding import HEContext
    return HEContext.from_params(small_ring())


def teacher(vocab, dim, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((vocab, dim), generator=g) / dim ** 0.5, 1 + 0.2 * torch.randn(dim, generator=g), g


@pytest.mark.parametrize("rows,vocab,dim,k", [(1, 10, 64, 3), (5, 1000, 192, 16), (40, 4099, 130, 8), (150, 700, 512, 100)])
@pytest.mark.parametrize("fast", [False, True])
def test_head(ctx, rows, vocab, dim, k, fast):
    """An operand of code c with scale s is off by at most 2^-4 of itself, or by 2^-10 s where codes run out of exponents (a block's largest number
    is at code 448, whose step is 32, half of it 2^-4 of 256 or more); a fast sum loses at most 2^-13 of its group's largest product from each."""
    from paper_2302_02407_amd.distill import TeacherHead
    table, weight, g = teacher(vocab, dim, rows)
    x, r = torch.randn((rows, dim), generator=g), torch.randn((rows, dim), generator=g)
    head = TeacherHead(ctx, table.cuda(), weight.cuda(), rows + 3, k, 2.0, dtype=torch.float32, fast_sums=fast)
    total = torch.empty((rows, dim), device="cuda")
    answers = head(x.cuda(), r.cuda(), total)
    assert torch.equal(total.cpu(), x + r)
    a, sa = R.norm(x, r, weight, 1e-6)
    w, sw = table.double(), head.table_scales.cpu()
    ea, ew = a.abs() * 2.0 ** -4 + R.spread(sa, dim) * 2.0 ** -10, w.abs() * 2.0 ** -4 + R.spread(sw.repeat_interleave(128, dim=0)[:vocab], dim) * 2.0 ** -10
    bound = 1.001 * (ea @ w.abs().T + a.abs() @ ew.T + ea @ ew.T) + (dim + 8) * 2.0 ** -24 * (a.abs() @ w.abs().T)
    if fast:
        kb = sa.shape[1]
        most = torch.stack([a[:, 128 * b:128 * b + 128].abs().amax(dim=1, keepdim=True) * w[:, 128 * b:128 * b + 128].abs().amax(dim=1) for b in range(kb)]).sum(dim=0)
        bound += 1.2 * 128 * 2.0 ** -13 * most
    z = head.logits[:rows].cpu()
    assert ((z.double() - a @ w.T).abs() <= bound).all()
    values, index, rest = R.top(z, k, 2.0)
    assert torch.equal(answers.index.cpu().long(), index) and torch.equal(answers.values.cpu().double(), values)
    assert ((answers.rest.cpu().double() - rest).abs() <= 2.0 ** -18 * (1 + rest.abs())).all()


def test_head_of_fewer_rows_and_refusals(ctx):
    from paper_2302_02407_amd.distill import TeacherHead, distill_loss
    table, weight, g = teacher(300, 256, 5)
    x = torch.randn((8, 256), generator=g).cuda()
    head = TeacherHead(ctx, table.cuda(), weight.cuda(), 8, 4, 1.0)
    whole, part = head(x), head(x[2:5])
    for a, b in zip(whole, part):
        assert torch.equal(a[2:5], b)
    with pytest.raises(ValueError):
        head(torch.zeros((9, 256), device="cuda"))
    with torch.cuda.stream(torch.cuda.Stream()):
        with pytest.raises(ValueError):
            head(x)
        with pytest.raises(ValueError):
            distill_loss(ctx, torch.zeros((8, 300), device="cuda"), whole, 1.0)


@pytest.mark.parametrize("alpha", [0.0, 0.3])
def test_descent_of_a_linear_student(ctx, alpha):
    """By a row's logits the loss has second derivatives of at most 1 in norm (a softmax's covariance is at most 1/2, there are two of them); by the
    weights of a linear student on features X, the mean loss of n rows has at most L = |X|^2 / n.  A step of 1/L then lowers it by |gradient|^2 / 2L."""
    from paper_2302_02407_amd.distill import TeacherHead, distill_loss
    n, vocab, dim, tau = 64, 500, 96, 2.0
    table, weight, g = teacher(vocab, dim, 9)
    x = torch.randn((n, dim), generator=g).cuda()
    answers = TeacherHead(ctx, 4 * table.cuda(), weight.cuda(), n, 24, tau)(x)
    labels = answers.index[:, 0].clone() if alpha else None
    w = torch.zeros((vocab, dim), device="cuda", requires_grad=True)
    most = float(torch.linalg.matrix_norm(x.double(), 2) ** 2 / n)
    last = None
    for _ in range(30):
        loss = distill_loss(ctx, x @ w.T, answers, tau, labels, alpha).mean()
        grad, = torch.autograd.grad(loss, w)
        now = float(loss.detach())
        assert last is None or now <= last + 1e-4 * abs(last) * 2.0 ** -4
        last = now - float(grad.double().square().sum()) / (2 * most)
        with torch.no_grad():
            w -= grad / most
    assert 0 < now


def test_student_learns_and_runs_on_a_ciphertext(ctx):
    """A student of one convolution, p(u) = 1.5 u - 0.5 u^3, the mean over the image and a linear layer: its gradients against 64 bits, some steps of
    training, and the trained convolution on an encrypted image."""
    from gpu_util import dev, host, zeros
    from oracle import ckks_client as K
    from oracle import conv2d as CV
    from oracle.he_oracle import Oracle
    from paper_2302_02407_amd.distill import TeacherHead, distill_loss
    n, vocab, dim, tau, alpha = 32, 50, 128, 2.0, 0.25
    table, weight, g = teacher(vocab, dim, 3)
    hidden, images = torch.randn((n, dim), generator=g), torch.randn((n, 4, 4, 4), generator=g)
    answers = TeacherHead(ctx, 4 * table.cuda(), weight.cuda(), n, 8, tau)(hidden.cuda())
    labels = answers.index[:, 0].clone()
    conv, linear = 0.1 * torch.randn((16, 4, 3, 3), generator=g), 0.3 * torch.randn((vocab, 16), generator=g)

    def student(x, conv, linear):
        patches = F.unfold(x, 3, padding=1)                              # one product: the same sums on either device
        u = (conv.flatten(1) @ patches).view(-1, 16, 4, 4)
        return (1.5 * u - 0.5 * u ** 3).mean(dim=(2, 3)) @ linear.T

    on_cpu = [t.double().requires_grad_() for t in (conv, linear)]
    z = student(images.double(), *on_cpu)
    want, dz, _ = R.distill(z.detach(), *(t.cpu() for t in answers), tau, labels.cpu(), alpha)
    z.backward(dz / n)
    on_gpu = [t.cuda().requires_grad_() for t in (conv, linear)]
    best = torch.optim.Adam(on_gpu, lr=0.02)
    losses = []
    for step in range(40):
        loss = distill_loss(ctx, student(images.cuda(), *on_gpu), answers, tau, labels, alpha).mean()
        best.zero_grad()
        loss.backward()
        losses.append(float(loss.detach()))
        if step == 0:
            assert abs(losses[0] - float(want.mean())) <= 1e-4 * float(want.mean())
            for a, b in zip(on_gpu, on_cpu):
                assert (a.grad.cpu().double() - b.grad).norm() <= 1e-4 * b.grad.norm()
        best.step()
    assert losses[-1] < losses[0]

    prm = small_ring()
    rng = S.make_rng(prm.seed)
    orc = Oracle.from_params(prm)
    cl = K.Client(orc, S.ternary_secret(rng, prm.N, prm.hamming))
    geo, level = CV.ConvGeometry(prm.N, 4, 4, 4, 16), 2
    for st in sorted(set(s for s in geo.tap_steps if s) | set(geo.ras_steps)):
        ctx.he_evk_register(ctx.galois_elt(st), dev(cl.rotation_key(orc.galois_elt(st), S.uniform_limbs(rng, prm.moduli, prm.N, prm.dnum),
                                                                    S.gaussian_error(rng, prm.N, prm.sigma, prm.dnum))))
    x, wt = images[0].double().numpy(), on_gpu[0].detach().cpu().double().numpy()
    ct = cl.encrypt(geo.pack_input(x).astype(np.complex128), prm.scale, level, S.uniform_limbs(rng, prm.q[:level + 1], prm.N)[0],
                    S.gaussian_error(rng, prm.N, prm.sigma)[0])
    pts = CV.encode_weights(orc, geo, wt, level, float(prm.q[level]))
    outs = [zeros(2, level, prm.N) for _ in range(geo.n_out)]
    ctx.he_conv2d(geo.C_a, geo.H, geo.W, geo.R, 3, level, [dev(pts[o, t]) for o in range(geo.n_out) for t in range(len(geo.taps))], dev(ct), outs)
    got, _ = geo.unpack_output([cl.decrypt(host(o), level - 1, prm.scale) for o in outs])
    assert np.max(np.abs(got - CV.conv2d_float(x, wt))) < 1e-3
