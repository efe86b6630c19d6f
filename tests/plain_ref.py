"""The plaintext operators (a teacher's head and a student's loss) from their definitions, in 64 bits on the CPU."""
import math

import torch

F8, F8_MAX, BLOCK = torch.float8_e4m3fn, 448.0, 128
ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # unit roundoff: 24, 8 and 11 significant bits


def matrix(rows, cols, dtype, pitch=None, offset=0, fill=math.nan):
    """A matrix on the GPU whose rows lie `pitch` elements apart, starting `offset` elements into its memory; what lies between is `fill`."""
    pitch = cols if pitch is None else pitch
    room = torch.empty(offset + rows * pitch + 16, dtype=dtype, device="cuda")
    (room.view(torch.uint8) if dtype == F8 else room).fill_(0x7f if dtype == F8 else fill)
    return room[offset:offset + rows * pitch].view(rows, pitch)[:, :cols]


def on_gpu(t, pitch=None, offset=0, fill=math.nan):
    return matrix(t.shape[0], t.shape[1], t.dtype, pitch, offset, fill).copy_(t.cuda())


def code_rows(t, more=0):
    """Codes on the GPU, rows at multiples of 16 bytes, NaN codes between them."""
    return on_gpu(t, -(-t.shape[1] // 16) * 16 + 16 * more)


def norm(x, residual, weight, eps):
    h = x.double() if residual is None else x.double() + residual.double()
    y = h / torch.sqrt(h.square().mean(dim=1, keepdim=True) + eps)
    y = y if weight is None else y * weight.double()
    scales = torch.stack([b.abs().amax(dim=1) for b in y.split(BLOCK, dim=1)], dim=1) / F8_MAX
    return y, scales


def spread(scales, cols):
    """One scale for each column."""
    return scales.double().repeat_interleave(BLOCK, dim=1)[:, :cols]


def product(a, sa, w, sw):
    """(A W^T, sum |A| |W|)"""
    x = a.double() * spread(sa, a.shape[1])
    y = w.double() * spread(sw.repeat_interleave(BLOCK, dim=0)[:w.shape[0]], w.shape[1])
    return x @ y.T, x.abs() @ y.abs().T


def top(z, k, tau):
    zd = z.double()
    rows = []
    for x in zd.tolist():                                      # a NaN stands above infinity
        rows.append(sorted(range(len(x)), key=lambda i: (x[i] == x[i], -x[i] if x[i] == x[i] else 0.0, i))[:k])
    index = torch.tensor(rows)
    rest = torch.logsumexp((zd / tau).scatter(1, index, -math.inf), dim=1)
    return zd.gather(1, index), index, rest


def distill(z, values, index, rest, tau, labels, alpha):
    """(loss, gradient of each row's loss by z, the sum of what the gradient's terms amount to), row by row as defined."""
    rows, vocab = z.shape
    loss, grad, size = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, vocab, dtype=torch.float64), torch.zeros(rows, vocab, dtype=torch.float64)
    for r in range(rows):
        x = z[r].double()
        y = None if labels is None else int(labels[r])
        if (y is not None and y < 0) or bool((x == -math.inf).all()):
            continue
        entries = [(int(i), float(v) / tau) for i, v in zip(index[r], values[r]) if 0 <= int(i) < vocab]
        t = torch.tensor([v for _, v in entries] + [-math.inf if rest is None else float(rest[r])], dtype=torch.float64)
        logq, kl = torch.log_softmax(x / tau, dim=0), 0.0
        q = logq.exp()
        if bool((t > -math.inf).any()):
            logp = torch.log_softmax(t, dim=0)
            p = logp.exp()
            named = torch.zeros(vocab, dtype=torch.bool)
            named[[i for i, _ in entries]] = True
            for j, (i, _) in enumerate(entries):
                if p[j] > 0:
                    kl += float(p[j] * (logp[j] - logq[i]))
                grad[r, i] -= p[j]
                size[r, i] += p[j]
            other = torch.where(named, -math.inf, logq)
            if p[-1] > 0:
                lr = torch.logsumexp(other, dim=0)
                kl += float(p[-1] * (logp[-1] - lr))
                share = torch.zeros_like(q) if lr == -math.inf else torch.where(named, 0.0, (other - lr).exp())
                grad[r] -= p[-1] * share
                size[r] += p[-1] * share
            grad[r] += q
            size[r] += q
            grad[r] *= (1 - alpha) * tau
            size[r] *= (1 - alpha) * tau
            if alpha < 1:
                loss[r] += (1 - alpha) * tau ** 2 * kl
        if y is not None and alpha > 0 and y < vocab:
            log1 = torch.log_softmax(x, dim=0)
            loss[r] -= alpha * log1[y]
            grad[r] += alpha * log1.exp()
            size[r] += alpha * log1.exp()
            grad[r, y] -= alpha
            size[r, y] += alpha
    return loss, grad, size
