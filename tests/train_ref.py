"""The operators of a training step from their definitions, in 64 bits on the CPU."""
import math

import torch

from plain_ref import BLOCK, F8, F8_MAX, ULP

LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}     # half of it is what a rounding can lose of a tiny number
PAIRS = [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, torch.float32), (torch.float16, torch.float32)]


def rng(seed):
    return torch.Generator().manual_seed(seed)


def untouched(t):
    """Whether what lies around the rows of a matrix made by plain_ref is still NaN."""
    around = torch.empty(0, dtype=t.dtype, device="cuda").set_(t.untyped_storage())
    return int(around.isnan().sum()) - int(t.isnan().sum()) == around.numel() - t.numel()


def rounding(x, dtype):
    """What storing x once may lose."""
    return x.abs() * ULP[dtype] * 1.001 + LEAST[dtype]


# ---- layer norm

def norm(h, eps):
    """(n, 1/sigma) of rows, 0 where there is nothing to divide by."""
    d = h.double() - h.double().mean(dim=1, keepdim=True)
    v = d.square().mean(dim=1, keepdim=True) + eps
    r = torch.where(v < 2.0 ** -120, 0.0, v.rsqrt())
    return d * r, r


def norm_grad(h, dy, weight, dsum, eps):
    """(dx, dweight, dbias, and what bounds the errors of each: sums of magnitudes)"""
    n, r = norm(h, eps)
    d = dy.double()
    g = d if weight is None else d * weight.double()
    mean = lambda x: x.mean(dim=1, keepdim=True)  # noqa: E731
    dx = r * (g - mean(g) - n * mean(g * n))
    size = r * (g.abs() + mean(g.abs()) + (1 + n.abs()) * mean(g.abs() * (1 + n.abs())))
    if dsum is not None:
        dx, size = dx + dsum.double(), size + dsum.double().abs()
    return dx, (d * n).sum(dim=0), d.sum(dim=0), size, (d.abs() * (1 + n.abs())).sum(dim=0), d.abs().sum(dim=0)


# ---- what is kept in 8 bits

def keep(u):
    """(codes, bytes) of rows."""
    codes, bytes_ = [], []
    for part in u.double().split(BLOCK, dim=1):
        most = part.abs().amax(dim=1)
        fine = most < math.inf
        e = torch.full_like(most, -110.0)
        some = fine & (most > 0)
        e[some] = torch.maximum(e[some], torch.ceil(torch.log2(most[some] / F8_MAX)))
        for _ in range(2):                                    # a logarithm is off by its rounding
            e = torch.where(some & (F8_MAX * 2.0 ** (e - 1) >= most) & (e > -110), e - 1, e)
        for _ in range(2):
            e = torch.where(some & (F8_MAX * 2.0 ** e < most), e + 1, e)
        e = torch.where(most == 0, -9.0, e)                   # zeros
        scaled = part / (2.0 ** e)[:, None]
        codes.append(torch.where(fine[:, None], scaled.float().to(F8).float(), math.nan).to(F8))
        bytes_.append(torch.where(fine, e + 127, 255.0).to(torch.uint8))
    return torch.cat(codes, dim=1), torch.stack(bytes_, dim=1)


def kept(codes, bytes_):
    """The numbers that these stand for."""
    power = torch.where(bytes_ == 255, math.nan, 2.0 ** (bytes_.double() - 127))
    return codes.float().double() * power.repeat_interleave(BLOCK, dim=1)[:, :codes.shape[1]]


def poly(u, coefs):
    """(y, the sum of its terms' magnitudes)"""
    u, powers = u.double(), range(len(coefs))
    return sum(float(coefs[i]) * u ** i for i in powers), sum(abs(float(coefs[i])) * u.abs() ** i for i in powers)


def poly_grad(v, coefs, dy):
    """(du, dcoefs, and the sums of magnitudes that bound their errors)"""
    d, n = dy.double(), len(coefs)
    slope = sum((i * float(coefs[i]) * v ** (i - 1) for i in range(1, n)), torch.zeros_like(v))
    size = sum((i * abs(float(coefs[i])) * v.abs() ** (i - 1) for i in range(1, n)), torch.zeros_like(v))
    return d * slope, torch.stack([(d * v ** i).sum() for i in range(n)]), d.abs() * size, torch.stack([(d * v ** i).abs().sum() for i in range(n)])


# ---- log probabilities

def distribution(z, tau):
    """(log p, p, entropy) of rows; a logit of -2^126 min(1, tau) or below is -infinity; rows of nothing else have no p and entropy 0."""
    x = z.double()
    x = torch.where(x <= -2.0 ** 126 * min(1.0, tau), -math.inf, x) / tau
    none = (x == -math.inf).all(dim=1, keepdim=True)
    logp = torch.where(none, -math.inf, torch.log_softmax(torch.where(none, 0.0, x), dim=1))
    p = logp.exp()
    return logp, p, -torch.where(p > 0, p * logp, 0.0).sum(dim=1)


def top_order(z, k):
    """Indices of the k largest of rows, the lowest first among equals, NaN above all."""
    rows = []
    for x in z.double().tolist():
        rows.append(sorted(range(len(x)), key=lambda i: (x[i] == x[i], -x[i] if x[i] == x[i] else 0.0, i))[:k])
    return torch.tensor(rows, dtype=torch.long).view(z.shape[0], k)


def logprobs_grad(z, tau, tokens, a, b):
    """(gradient, what its terms amount to).  A power of two below 2^-126 may count as 0 (the instruction's results are normal numbers): then a
    probability, which is such a power over a sum of at least 1, is off by 2^-126, and what it is multiplied by off by as much; a bound takes 2e-5 of the size."""
    logp, p, entropy = distribution(z, tau)
    rows, vocab = z.shape
    grad, size = torch.zeros(rows, vocab, dtype=torch.float64), torch.zeros(rows, vocab, dtype=torch.float64)
    for r in range(rows):
        y = -1 if tokens is None else int(tokens[r])
        wa = float(a[r]) if a is not None and 0 <= y < vocab and (p[r] > 0).any() else 0.0
        wb = float(b[r]) if b is not None else 0.0
        lp = torch.where(p[r] > 0, logp[r], 0.0)
        grad[r] = -(wa * p[r] + wb * p[r] * (lp + entropy[r])) / tau
        size[r] = (p[r] + 2.0 ** -126 / 2e-5 * (p[r] > 0)) * (abs(wa) + abs(wb) * (1 + lp.abs() + entropy[r])) / tau
        if wa:
            grad[r, y] += wa / tau
            size[r, y] += abs(wa) / tau
    return grad, size
