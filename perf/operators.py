"""The plaintext side of a network that is to be evaluated encrypted, as timed cases: a teacher's head and a student's loss.

A network of low-degree activations is trained by distillation before its filters are encoded: a teacher that need not be
friendly to encryption runs in 8 bits (its last residual addition and norm, and the product with its class or vocabulary
weights), its top logits are kept, and the student's logits are held against them.  Four operators, each through the
public binding (`paper_2302_02407_amd.binding.HEContext`):

  norm     residual addition, root-mean-square norm, output in 8 bits with one scale for each 128 values
  product  matrix product of 8-bit codes with a scale for each block of 128 (weights: of 128 x 128)
  top      a row's k largest logits in order, and the log-sum-exp of the rest at a temperature
  distill  the distillation loss against those, mixed with the label's cross entropy, and its gradient; in one call
           (`step`) or as a loss and, later, its gradient (`later`)

8 bits are e4m3 (largest value 448).  Rows of codes start at multiples of 16 bytes.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
F8, F8_MAX, BLOCK = torch.float8_e4m3fn, 448.0, 128
EPS = 1e-5


def listed():
    return [
        # one token of a teacher that answers as it writes: latency alone
        {"name": "norm_one_token", "kind": "norm", "rows": 1, "dim": 4096, "dtype": "bf16", "residual": True, "weight": True},
        # a ragged batch of an odd width with neither a residual nor a weight
        {"name": "norm_odd_width", "kind": "norm", "rows": 517, "dim": 1001, "dtype": "f16", "residual": False, "weight": False},
        # the tokens of a training step's batch: streaming
        {"name": "norm_batch", "kind": "norm", "rows": 16384, "dim": 4096, "dtype": "bf16", "residual": True, "weight": True},
        # one token against a vocabulary: the weights are read once, nothing else counts
        {"name": "product_one_token", "kind": "product", "m": 1, "n": 32768, "k": 4096, "out": "bf16"},
        # a few images against 1000 classes: too little work to fill the card
        {"name": "product_classes", "kind": "product", "m": 24, "n": 1000, "k": 2048, "out": "f32"},
        # sizes that no tile divides, the last block of the sum a partial one
        {"name": "product_odd", "kind": "product", "m": 777, "n": 10007, "k": 2040, "out": "f16"},
        # a training step's tokens against a vocabulary: matrix arithmetic
        {"name": "product_batch", "kind": "product", "m": 8192, "n": 32768, "k": 4096, "out": "bf16"},
        # a batch of images, 1000 classes
        {"name": "top_classes", "kind": "top", "rows": 256, "vocab": 1000, "k": 20, "tau": 4.0, "dtype": "f32"},
        # a training step's tokens, a large vocabulary: one pass over the logits
        {"name": "top_batch", "kind": "top", "rows": 2048, "vocab": 131072, "k": 64, "tau": 2.0, "dtype": "bf16"},
        # a batch of images, 1000 classes, labels beside the teacher
        {"name": "distill_classes", "kind": "distill", "rows": 256, "vocab": 1000, "k": 20, "tau": 4.0, "alpha": 0.1, "rest": True, "labels": True, "step": True, "dtype": "f32"},
        # an odd vocabulary whose rows start anywhere; the gradient is asked for later, as automatic differentiation does
        {"name": "distill_odd_later", "kind": "distill", "rows": 1031, "vocab": 50021, "k": 33, "tau": 1.0, "alpha": 0.5, "rest": False, "labels": True, "step": False, "dtype": "bf16"},
        # a training step's tokens, a large vocabulary, loss and gradient in one call
        {"name": "distill_batch", "kind": "distill", "rows": 4096, "vocab": 131072, "k": 64, "tau": 2.0, "alpha": 0.0, "rest": True, "labels": False, "step": True, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 2e15 if c["kind"] == "product" else 0.0)


def draw(rng):
    """One more case of these kinds; none costs more than the largest listed one of its kind."""
    kind = rng.choice(["norm", "product", "product", "top", "distill", "distill"])
    most = max(_cost(c) for c in listed() if c["kind"] == kind)
    while True:
        c = _draw(rng, kind)
        if _cost(c) <= most:
            return c


def _draw(rng, kind):
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "norm":
        return {"kind": kind, "rows": _log_int(rng, 1, 16384), "dim": _log_int(rng, 64, 16384), "dtype": dtype, "residual": rng.random() < 0.7, "weight": rng.random() < 0.8}
    if kind == "product":
        return {"kind": kind, "m": _log_int(rng, 1, 8192), "n": _log_int(rng, 10, 131072), "k": _log_int(rng, 64, 16384), "out": dtype}
    vocab = _log_int(rng, 10, 131072)
    c = {"kind": kind, "rows": _log_int(rng, 1, 8192), "vocab": vocab, "k": _log_int(rng, 1, min(vocab, 128)), "tau": rng.choice([1.0, 1.5, 2.0, 4.0])}
    if kind == "distill":
        c |= {"alpha": rng.choice([0.0, 0.1, 0.5]), "rest": rng.random() < 0.6, "labels": rng.random() < 0.6, "step": rng.random() < 0.6}
        c["alpha"] = c["alpha"] if c["labels"] else 0.0
    return c | {"dtype": dtype}


def work(case):
    c = case
    if c["kind"] == "norm":
        n, es = c["rows"] * c["dim"], SIZE[c["dtype"]]
        return {"bytes": n * (es * (3 if c["residual"] else 1) + 1) + 4 * c["rows"] * -(-c["dim"] // BLOCK) + (es * c["dim"] if c["weight"] else 0), "flops": 6 * n}
    if c["kind"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        kb = -(-k // BLOCK)
        return {"bytes": (m + n) * k + 4 * kb * (m + -(-n // BLOCK)) + m * n * SIZE[c["out"]], "flops": 2 * m * n * k}
    rows, n = c["rows"], c["rows"] * c["vocab"]
    if c["kind"] == "top":
        return {"bytes": n * SIZE[c["dtype"]] + rows * (8 * c["k"] + 4), "flops": 3 * n}
    small = rows * (8 * c["k"] + 4 + 4 + (4 if c["rest"] else 0) + (4 if c["labels"] else 0))
    return {"bytes": 2 * n * SIZE[c["dtype"]] + small, "flops": 10 * n}


# ---- inputs

def _padded(rows, dim):
    """Room for rows of codes that start at multiples of 16 bytes."""
    return torch.zeros((rows, -(-dim // 16) * 16), dtype=torch.uint8, device="cuda").view(F8)[:, :dim]


def _codes(x, rows_per_scale):
    """Codes of x and their scales: one for each 128 columns of `rows_per_scale` rows."""
    rows, dim = x.shape
    rb, kb = -(-rows // rows_per_scale), -(-dim // BLOCK)
    p = torch.zeros((rb * rows_per_scale, kb * BLOCK), device=x.device)
    p[:rows, :dim] = x
    p = p.view(rb, rows_per_scale, kb, BLOCK)
    scale = p.abs().amax(dim=(1, 3)).clamp_min(1e-12) / F8_MAX
    q = (p / scale[:, None, :, None]).view(rb * rows_per_scale, kb * BLOCK)[:rows, :dim].to(F8)
    out = _padded(rows, dim)
    out.copy_(q)
    return out, scale.contiguous()


def _logits(g, rows, vocab, dtype):
    """Logits as networks give them: a broad bulk, some classes that stand out, and padding of a vocabulary masked out."""
    z = torch.randn((rows, vocab), generator=g, device="cuda") * 2
    few = min(32, max(1, vocab // 8))
    at, high = torch.randint(0, vocab, (rows, few), generator=g, device="cuda"), 5 + 9 * torch.rand((rows, few), generator=g, device="cuda")
    z.scatter_reduce_(1, at, high, "amax")
    if vocab > 512:
        z[:, vocab - vocab // 64:] = -math.inf
    return z.to(DTYPES[dtype])


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c, "ctx": _context() if own else None}
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if c["kind"] == "norm":
        rows, dim, t = c["rows"], c["dim"], DTYPES[c["dtype"]]
        spread = torch.exp(0.7 * torch.randn(dim, generator=g, device="cuda"))          # a few loud channels
        s["x"] = (torch.randn((rows, dim), generator=g, device="cuda") * spread).to(t)
        s["residual"] = (4 * torch.randn((rows, dim), generator=g, device="cuda") * spread).to(t) if c["residual"] else None
        s["weight"] = (1 + 0.2 * torch.randn(dim, generator=g, device="cuda")).to(t) if c["weight"] else None
        s["sum"] = new(rows, dim, dtype=t) if c["residual"] else None
        s["codes"], s["scales"] = _padded(rows, dim), new(rows, -(-dim // BLOCK))
        return s
    if c["kind"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        s["a"], s["a_scales"] = _codes(torch.randn((m, k), generator=g, device="cuda") * torch.exp(0.5 * torch.randn(k, generator=g, device="cuda")), 1)
        s["w"], s["w_scales"] = _codes(torch.randn((n, k), generator=g, device="cuda") / math.sqrt(k), BLOCK)
        s["out"] = new(m, n, dtype=DTYPES[c["out"]])
        return s
    rows, vocab, k = c["rows"], c["vocab"], c["k"]
    s["z"] = _logits(g, rows, vocab, c["dtype"])
    s["values"], s["index"], s["rest"] = new(rows, k), new(rows, k, dtype=torch.int32), new(rows)
    if c["kind"] == "top":
        return s
    for lo in range(0, rows, 512):                # the teacher agrees with the student in part
        z = s["z"][lo:lo + 512].float()
        z = 0.8 * z + 1.5 * torch.randn(z.shape, generator=g, device="cuda")
        v, i = z.topk(k, dim=1)
        s["values"][lo:lo + 512], s["index"][lo:lo + 512] = v, i.to(torch.int32)
        s["rest"][lo:lo + 512] = torch.logsumexp(z.scatter_(1, i, -math.inf) / c["tau"], dim=1)
        del z
    s["index"][rows // 2, k // 2:] = -1           # a row for which the teacher gave fewer
    if not c["rest"]:
        s["rest"] = None
    s["labels"] = None
    if c["labels"]:
        s["labels"] = torch.randint(0, vocab - vocab // 64, (rows,), generator=g, device="cuda", dtype=torch.int32)
        s["labels"][torch.rand(rows, generator=g, device="cuda") < 0.06] = -1          # padding between texts
    # the mean over the rows; gradients in f16 are scaled up, as its small range needs it
    s["weights"] = torch.full((rows,), (4096.0 if c["dtype"] == "f16" else 1.0) / rows, device="cuda")
    s["loss"], s["stats"], s["grad"] = new(rows), new(rows, 4), torch.empty_like(s["z"])
    return s


# ---- one pass

_made = []


def _context():
    """The handle that a program keeps: made once."""
    if not _made:
        from he_inputs.params import config_params
        from paper_2302_02407_amd.binding import HEContext
        _made.append(HEContext.from_params(config_params(0)))
    return _made[0]


def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c, s["ctx"])
    return {"norm": _norm, "product": _product, "top": _top, "distill": _distill}[c["kind"]](s, c)


def _own(s, c, ctx):
    if c["kind"] == "norm":
        ctx.he_rmsnorm_q8(s["x"], s["codes"], s["scales"], EPS, residual=s["residual"], weight=s["weight"], sum_out=s["sum"])
        return {"codes": s["codes"], "scales": s["scales"], "sum": s["sum"]}
    if c["kind"] == "product":
        ctx.he_matmul_q8(s["a"], s["a_scales"], s["w"], s["w_scales"], s["out"], fast_sums=c["out"] != "f32")   # what is rounded to 16 bits needs no exact sums
        return {"out": s["out"]}
    if c["kind"] == "top":
        ctx.he_top_logits(s["z"], c["tau"], s["values"], s["index"], s["rest"])
        return {"values": s["values"], "index": s["index"], "rest": s["rest"]}
    teacher = (s["values"], s["index"], s["rest"])
    if c["step"]:
        ctx.he_distill_loss(s["z"], *teacher, c["tau"], s["loss"], labels=s["labels"], alpha=c["alpha"], grad=s["grad"], row_weights=s["weights"])
    else:
        ctx.he_distill_loss(s["z"], *teacher, c["tau"], s["loss"], labels=s["labels"], alpha=c["alpha"], stats=s["stats"])
        ctx.he_distill_grad(s["z"], *teacher, c["tau"], s["stats"], s["weights"], s["grad"], labels=s["labels"], alpha=c["alpha"])
    return {"loss": s["loss"], "grad": s["grad"]}


def _norm(s, c):
    t, dim = DTYPES[c["dtype"]], c["dim"]
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS)
    if s["weight"] is not None:
        y = y * s["weight"].float()
    kb = -(-dim // BLOCK)
    y = torch.nn.functional.pad(y, (0, kb * BLOCK - dim)).view(-1, kb, BLOCK)
    scales = y.abs().amax(dim=2) / F8_MAX
    codes = (y / scales.clamp_min(1e-37)[:, :, None]).view(-1, kb * BLOCK)[:, :dim].to(F8)
    return {"codes": codes, "scales": scales, "sum": h.to(t) if s["residual"] is not None else None}


def _product(s, c):
    k = c["k"]
    a = s["a"].float() * s["a_scales"].repeat_interleave(BLOCK, dim=1)[:, :k]
    w = s["w"].float() * s["w_scales"].repeat_interleave(BLOCK, dim=0)[:c["n"]].repeat_interleave(BLOCK, dim=1)[:, :k]
    return {"out": torch.matmul(a, w.t()).to(DTYPES[c["out"]])}


def _top(s, c):
    z = s["z"].float()
    bits = (z + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7fffffff) - 1, bits)       # in the order of the numbers
    at = torch.arange(c["vocab"], device=z.device)
    key = (key << 32) + (c["vocab"] - 1 - at)                         # the lowest index first among equals
    i = (c["vocab"] - 1) - (key.topk(c["k"], dim=1).values & 0xffffffff)
    values = z.gather(1, i)
    m = (z / c["tau"]).scatter(1, i, -math.inf)
    high = m.amax(dim=1, keepdim=True).clamp_min(-3e38)
    rest = (m - high).exp_().sum(dim=1).log() + high[:, 0]
    return {"values": values, "index": i.to(torch.int32), "rest": rest}


def _lse(x):
    high = x.amax(dim=1, keepdim=True).clamp_min(-3e38)
    return (x - high).exp_().sum(dim=1, keepdim=True).log() + high


def _shares(t, r):
    """Probabilities of the top and of the rest, and their logarithms: where the rest holds nearly all, one minus the top's share."""
    high = torch.maximum(t.amax(dim=1, keepdim=True), r).clamp_min(-3e38)
    et, er = (t - high).exp(), (r - high).exp()
    top = et.sum(dim=1, keepdim=True)
    return et / (top + er), er / (top + er), t - high - (top + er).log(), -torch.log1p(top / er)


def _distill(s, c):
    tau, alpha, rows = c["tau"], c["alpha"], c["rows"]
    z = s["z"].float()
    there = s["index"] >= 0
    at = s["index"].clamp_min(0).long()
    none = torch.full_like(s["values"], -math.inf)
    t = torch.where(there, s["values"] / tau, none)
    r = s["rest"][:, None] if c["rest"] else none[:, :1]
    pt, pr, logpt, logpr = _shares(t, r)
    x = z / tau
    hit = torch.zeros_like(x).scatter_add_(1, at, there.float()) > 0
    high = x.amax(dim=1, keepdim=True).clamp_min(-3e38)
    e = (x - high).exp_()
    top, other = torch.where(hit, e, 0.0).sum(dim=1, keepdim=True), torch.where(hit, 0.0, e).sum(dim=1, keepdim=True)
    logqt = x.gather(1, at) - high - (top + other).log()
    logqr = -torch.log1p(top / other)
    kl = torch.where(pt > 0, pt * (logpt - logqt), 0.0).sum(dim=1) + torch.where(pr > 0, pr * (logpr - logqr), 0.0)[:, 0]
    loss = (1 - alpha) * tau * tau * kl
    grad = e / (top + other)
    if c["rest"]:
        grad -= torch.where(hit, 0.0, e * (pr / other))
    grad.scatter_add_(1, at, torch.where(there, -pt, 0.0))
    grad *= (1 - alpha) * tau
    if s["labels"] is not None:
        live = (s["labels"] >= 0)
        y = s["labels"].clamp_min(0).long()[:, None]
        e = _lse(z)
        loss = torch.where(live, loss + alpha * (e - z.gather(1, y))[:, 0], 0.0)
        grad += alpha * (z - e).exp_()
        grad.scatter_add_(1, y, torch.full((rows, 1), -alpha, device=z.device))
        grad *= live[:, None]
    return {"loss": loss, "grad": (grad * s["weights"][:, None]).to(s["z"].dtype)}


# ---- from the definitions, in 64 bits

def exact(case, seed):
    c, s = case, prepare(case, seed)
    return {"norm": _exact_norm, "product": _exact_product, "top": _exact_top, "distill": _exact_distill}[c["kind"]](s, c)


def _exact_norm(s, c):
    out = {"codes": [], "scales": [], "sum": []}
    for lo in range(0, c["rows"], 4096):
        h = s["x"][lo:lo + 4096].double()
        if s["residual"] is not None:
            h = h + s["residual"][lo:lo + 4096].double()
        y = h / torch.sqrt(h.square().sum(1) / c["dim"] + EPS)[:, None]
        if s["weight"] is not None:
            y = y * s["weight"].double()
        parts = [p for p in y.split(BLOCK, dim=1)]
        scales = [p.abs().max(dim=1).values / F8_MAX for p in parts]
        out["codes"].append(torch.cat([torch.where(k[:, None] > 0, p / k[:, None], 0.0).to(F8).double() for p, k in zip(parts, scales)], dim=1))
        out["scales"].append(torch.stack(scales, dim=1))
        out["sum"].append(h)
    out = {k: torch.cat(v) for k, v in out.items()}
    return out if s["residual"] is not None else out | {"sum": None}


def _exact_product(s, c):
    if 2.0 * c["m"] * c["n"] * c["k"] > 3e12:
        return None
    out = torch.zeros((c["m"], c["n"]), dtype=torch.float64, device="cuda")
    for b in range(-(-c["k"] // BLOCK)):
        k = slice(b * BLOCK, min(c["k"], (b + 1) * BLOCK))
        part = s["a"][:, k].double() @ s["w"][:, k].double().t()
        for nb in range(s["w_scales"].shape[0]):
            part[:, nb * BLOCK:(nb + 1) * BLOCK] *= s["w_scales"][nb, b].double()
        out.addcmul_(part, s["a_scales"][:, b:b + 1].double())
        del part
    return {"out": out}


def _exact_top(s, c):
    values, index, rest = [], [], []
    for lo in range(0, c["rows"], 128):
        v, i = s["z"][lo:lo + 128].double().sort(dim=1, descending=True, stable=True)
        values.append(v[:, :c["k"]])
        index.append(i[:, :c["k"]].to(torch.int32))
        tail = v[:, c["k"]:] / c["tau"]
        rest.append(torch.logsumexp(tail, dim=1) if tail.shape[1] else torch.full((v.shape[0],), -math.inf, dtype=torch.float64, device=v.device))
    return {"values": torch.cat(values), "index": torch.cat(index), "rest": torch.cat(rest)}


def _exact_distill(s, c):
    tau, alpha, k, losses, grads = c["tau"], c["alpha"], c["k"], [], []
    for lo in range(0, c["rows"], 256):
        cut = slice(lo, lo + 256)
        z, at = s["z"][cut].double(), s["index"][cut].long()
        rows, vocab = z.shape
        given = at >= 0
        # the teacher's probabilities spread over the vocabulary; one column more takes what stands at no index
        t = torch.where(given, s["values"][cut].double() / tau, -math.inf)
        r = s["rest"][cut].double() if c["rest"] else torch.full((rows,), -math.inf, dtype=torch.float64, device="cuda")
        probs = torch.softmax(torch.cat([t, r[:, None]], dim=1), dim=1)
        p = torch.zeros((rows, vocab + 1), dtype=torch.float64, device="cuda").scatter_add_(1, torch.where(given, at, vocab), probs[:, :k])[:, :vocab]
        inside = torch.zeros((rows, vocab + 1), dtype=torch.bool, device="cuda").scatter_(1, torch.where(given, at, vocab), True)[:, :vocab]
        logq = torch.log_softmax(z / tau, dim=1)
        kl = torch.where(p > 0, torch.special.xlogy(p, p) - p * logq, 0.0).sum(1)
        grad = logq.exp() - p
        if c["rest"]:
            other = torch.where(inside, -math.inf, logq)
            all_other = torch.logsumexp(other, dim=1)
            kl = kl + torch.where(probs[:, k] > 0, torch.special.xlogy(probs[:, k], probs[:, k]) - probs[:, k] * all_other, 0.0)
            share = torch.where(torch.isinf(all_other)[:, None], 0.0, (other - all_other[:, None]).exp())
            grad = grad - probs[:, k:] * share
        loss, grad = (1 - alpha) * tau ** 2 * kl, (1 - alpha) * tau * grad
        if c["labels"]:
            y = s["labels"][cut].long()
            log1 = torch.log_softmax(z, dim=1)
            hot = torch.zeros_like(z).scatter_(1, y.clamp_min(0)[:, None], 1.0)
            loss = loss - alpha * log1.gather(1, y.clamp_min(0)[:, None])[:, 0]
            grad = grad + alpha * (log1.exp() - hot)
            loss, grad = torch.where(y >= 0, loss, 0.0), torch.where(y[:, None] >= 0, grad, 0.0)
        losses.append(loss)
        grads.append(grad * s["weights"][cut, None].double())
    return {"loss": torch.cat(losses), "grad": torch.cat(grads)}
