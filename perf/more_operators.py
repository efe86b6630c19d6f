"""A training step around the loss of a network that is to be evaluated encrypted, as timed cases.

Such a network and its teacher are trained in the clear.  Four operators of that step, each through the public binding
(`paper_2302_02407_amd.binding.HEContext`), forward or backward:

  norm    layer norm with a residual addition before it; backward: the gradient by the normed rows (with what comes down the
          residual path added) and by weight and bias
  act     the student's activation, a polynomial with trained coefficients, which keeps its input in 8 bits; backward from these:
          the gradient by the input and by the coefficients
  weight  the gradient of a linear layer's weight from its input as kept in 8 bits
  score   log probabilities of given tokens, entropy and the most probable alternatives; backward: the gradient by the logits

A row that is kept in 8 bits has e4m3 codes and, for each 128 columns, one byte b: a value is its code times 2^(b - 127), the smallest such
power from 2^-110 on at which the largest of the block is at most 448.  Rows of codes start at multiples of 16 bytes.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
F8, F8_MAX, BLOCK, LEAST = torch.float8_e4m3fn, 448.0, 128, -110
EPS = 1e-5


def listed():
    return [
        # one token of a model that answers as it writes: latency alone
        {"name": "norm_one_token", "kind": "norm", "grad": False, "rows": 1, "dim": 4096, "dtype": "bf16", "params": "bf16", "residual": True},
        # a ragged batch of an odd width, backward
        {"name": "norm_odd_grad", "kind": "norm", "grad": True, "rows": 517, "dim": 1001, "dtype": "f16", "params": "f16", "residual": False},
        # the tokens of a training step's batch, parameters kept in 32 bits, backward: streaming beside two sums over all rows
        {"name": "norm_batch_grad", "kind": "norm", "grad": True, "rows": 16384, "dim": 4096, "dtype": "bf16", "params": "f32", "residual": True},
        # a few images' features
        {"name": "act_images", "kind": "act", "grad": False, "rows": 24, "dim": 2048, "dtype": "f32", "degree": 3},
        # odd sizes, a polynomial of a higher degree, backward
        {"name": "act_odd_grad", "kind": "act", "grad": True, "rows": 777, "dim": 10007, "dtype": "f16", "degree": 7},
        # a training step's batch, backward: streaming
        {"name": "act_batch_grad", "kind": "act", "grad": True, "rows": 16384, "dim": 8192, "dtype": "bf16", "degree": 3},
        # a batch of images, the layer to 1000 classes
        {"name": "weight_classes", "kind": "weight", "m": 256, "n": 1000, "k": 2048, "dtype": "f32", "out": "f32"},
        # a long ragged batch, a small layer of odd sizes: the sum's axis is the long one
        {"name": "weight_odd", "kind": "weight", "m": 20011, "n": 777, "k": 1001, "dtype": "f16", "out": "f16"},
        # a training step's batch: matrix arithmetic
        {"name": "weight_batch", "kind": "weight", "m": 16384, "n": 8192, "k": 4096, "dtype": "bf16", "out": "f32"},
        # one token and its alternatives as it is written: one long row
        {"name": "score_one_token", "kind": "score", "grad": False, "rows": 1, "vocab": 131072, "k": 20, "tau": 1.0, "dtype": "bf16"},
        # the texts of a scoring batch: one pass over the logits
        {"name": "score_batch", "kind": "score", "grad": False, "rows": 2048, "vocab": 131072, "k": 8, "tau": 1.0, "dtype": "bf16"},
        # an odd vocabulary whose rows start anywhere, backward
        {"name": "score_odd_grad", "kind": "score", "grad": True, "rows": 2055, "vocab": 50021, "k": 1, "tau": 1.5, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 2e15 if c["kind"] == "weight" else 0.0)


def draw(rng):
    """One more case of these kinds; none costs more than the largest listed one of its kind."""
    kind = rng.choice(["norm", "act", "weight", "score"])
    most = max(_cost(c) for c in listed() if c["kind"] == kind)
    while True:
        c = _draw(rng, kind)
        if _cost(c) <= most:
            return c


def _draw(rng, kind):
    dtype, grad = rng.choice(["bf16", "bf16", "f16", "f32"]), rng.random() < 0.6
    if kind == "norm":
        return {"kind": kind, "grad": grad, "rows": _log_int(rng, 1, 65536), "dim": _log_int(rng, 16, 32768), "dtype": dtype, "params": rng.choice([dtype, "f32"]), "residual": rng.random() < 0.6}
    if kind == "act":
        return {"kind": kind, "grad": grad, "rows": _log_int(rng, 1, 65536), "dim": _log_int(rng, 16, 32768), "dtype": dtype, "degree": rng.randint(1, 8)}
    if kind == "weight":
        return {"kind": kind, "m": _log_int(rng, 1, 65536), "n": _log_int(rng, 10, 32768), "k": _log_int(rng, 16, 16384), "dtype": dtype, "out": rng.choice([dtype, "f32"])}
    vocab = _log_int(rng, 10, 131072)
    return {"kind": kind, "grad": grad, "rows": _log_int(rng, 1, 8192), "vocab": vocab, "k": _log_int(rng, 1, min(vocab, 128)), "tau": rng.choice([0.7, 1.0, 1.0, 2.0]), "dtype": dtype}


def work(case):
    c = case
    if c["kind"] == "norm":
        n, es, params = c["rows"] * c["dim"], SIZE[c["dtype"]], c["dim"] * SIZE[c["params"]]
        if c["grad"]:
            return {"bytes": n * es * (4 if c["residual"] else 3) + 16 * c["rows"] + 3 * params, "flops": 14 * n}
        return {"bytes": n * es * (4 if c["residual"] else 2) + 16 * c["rows"] + 2 * params, "flops": 8 * n}
    if c["kind"] == "act":
        n = c["rows"] * c["dim"]
        return {"bytes": n * (2 * SIZE[c["dtype"]] + 1) + c["rows"] * -(-c["dim"] // BLOCK) + 4 * (c["degree"] + 1) * (2 if c["grad"] else 1),
                "flops": n * c["degree"] * (6 if c["grad"] else 2)}
    if c["kind"] == "weight":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": m * n * SIZE[c["dtype"]] + m * (k + -(-k // BLOCK)) + n * k * SIZE[c["out"]], "flops": 2 * m * n * k}
    rows, n = c["rows"], c["rows"] * c["vocab"]
    if c["grad"]:
        return {"bytes": 2 * n * SIZE[c["dtype"]] + rows * (4 + 16 + 8), "flops": 8 * n}
    return {"bytes": n * SIZE[c["dtype"]] + rows * (4 + 8 + 16 + 8 * c["k"]), "flops": 6 * n}


# ---- inputs

def _padded(rows, dim):
    """Room for rows of codes that start at multiples of 16 bytes."""
    return torch.zeros((rows, -(-dim // 16) * 16), dtype=torch.uint8, device="cuda").view(F8)[:, :dim]


def _blocks(x):
    """Rows in blocks of 128 columns, filled up with zeros."""
    kb = -(-x.shape[1] // BLOCK)
    return torch.nn.functional.pad(x, (0, kb * BLOCK - x.shape[1])).view(x.shape[0], kb, BLOCK)


def _power(e):
    """2^e, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _kept(x):
    """What is kept of numbers of 32 bits: codes and the powers' bytes."""
    b = _blocks(x)
    fraction, exponent = torch.frexp(b.abs().amax(dim=2))          # the largest is fraction * 2^exponent, and 448 is 0.875 * 2^9
    e = (exponent - 9 + (fraction > F8_MAX / 512).int()).clamp_min(LEAST)
    codes = (b * _power(-e)[:, :, None]).view(x.shape[0], -1)[:, :x.shape[1]].to(F8)
    return codes, (e + 127).to(torch.uint8)


def _values(codes, exponents):
    """The numbers that codes and bytes stand for, in 32 bits: exact."""
    b = _blocks(codes.float()) * _power(exponents.int() - 127)[:, :, None]
    return b.view(codes.shape[0], -1)[:, :codes.shape[1]]


def _checkpoint(x):
    codes, exponents = _kept(x)
    out = _padded(*x.shape)
    out.copy_(codes)
    return out, exponents


def _logits(g, rows, vocab, dtype):
    """Logits as networks give them: a broad bulk, some tokens that stand out, and padding of a vocabulary masked out."""
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
    s = {"case": c}
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    up = 4096.0 if c["dtype"] == "f16" else 1.0        # gradients in f16 are scaled up, as its small range needs it
    t = DTYPES[c["dtype"]]
    if c["kind"] == "norm":
        rows, dim, p = c["rows"], c["dim"], DTYPES[c["params"]]
        spread = torch.exp(0.7 * normal(dim))          # a few loud channels, and a mean that is not 0
        x = ((normal(rows, dim) + 0.5) * spread).to(t)
        s["weight"], s["bias"] = (1 + 0.2 * normal(dim)).to(p), (0.1 * normal(dim)).to(p)
        if not c["grad"]:
            s["x"], s["residual"] = x, (4 * normal(rows, dim) * spread).to(t) if c["residual"] else None
            s["y"], s["sum"], s["stats"] = new(rows, dim, dtype=t), new(rows, dim, dtype=t) if c["residual"] else None, new(rows, 4)
            return s
        s["h"], s["dy"] = x, (up * 1e-3 * normal(rows, dim)).to(t)
        s["dsum"] = (up * 1e-3 * normal(rows, dim)).to(t) if c["residual"] else None
        h = x.double()
        var, mean = torch.var_mean(h, dim=1, unbiased=False)
        s["stats"] = torch.stack([mean.float(), (mean - mean.float()).float(), (var + EPS).rsqrt().float(), torch.zeros(rows, device="cuda")], dim=1)
        s["dx"], s["dweight"], s["dbias"] = new(rows, dim, dtype=t), new(dim, dtype=p), new(dim, dtype=p)
        return s
    if c["kind"] == "act":
        rows, dim, n = c["rows"], c["dim"], c["degree"] + 1
        u = (normal(rows, dim) * torch.exp(0.3 * normal(rows, 1))).clamp_(-6, 6)
        u[torch.rand(rows, generator=g, device="cuda") < 0.06] = 0                             # padding between texts
        s["coefs"] = normal(n) / torch.tensor([float(math.factorial(i)) for i in range(n)], device="cuda")
        if not c["grad"]:
            s["u"], s["y"], s["codes"], s["exponents"] = u.to(t), new(rows, dim, dtype=t), _padded(rows, dim), new(rows, -(-dim // BLOCK), dtype=torch.uint8)
            return s
        s["codes"], s["exponents"] = _checkpoint(u.to(t).float())
        s["dy"], s["du"], s["dcoefs"] = (up * 1e-3 * normal(rows, dim)).to(t), new(rows, dim, dtype=t), new(n)
        return s
    if c["kind"] == "weight":
        m, n, k = c["m"], c["n"], c["k"]
        s["codes"], s["exponents"] = _checkpoint(normal(m, k) * torch.exp(0.5 * normal(m, 1)) * torch.exp(0.3 * normal(k)))
        s["dy"] = (up * 1e-3 * normal(m, n) * (torch.rand((m, 1), generator=g, device="cuda") > 0.06 if m > 16 else 1.0)).to(t)   # padding between texts
        s["dw"] = new(n, k, dtype=DTYPES[c["out"]])
        return s
    rows, vocab, k = c["rows"], c["vocab"], c["k"]
    s["z"] = _logits(g, rows, vocab, c["dtype"])
    s["tokens"] = torch.randint(0, vocab - vocab // 64, (rows,), generator=g, device="cuda", dtype=torch.int32)
    likely = torch.rand(rows, generator=g, device="cuda") < 0.7
    s["tokens"] = torch.where(likely, s["z"].argmax(dim=1).to(torch.int32), s["tokens"])
    s["tokens"][torch.rand(rows, generator=g, device="cuda") < (0.06 if rows > 16 else 0.0)] = -1       # padding between texts
    if not c["grad"]:
        s["logp"], s["entropy"], s["values"], s["index"], s["stats"] = new(rows), new(rows), new(rows, k), new(rows, k, dtype=torch.int32), new(rows, 4)
        return s
    s["stats"] = torch.zeros((rows, 4), device="cuda")
    for lo in range(0, rows, 512):                     # what the forward pass left: the largest logit, the sum against it, the entropy
        z = s["z"][lo:lo + 512].double()
        high = z.amax(dim=1)
        x = (z - high[:, None]) / c["tau"]
        e = x.exp()
        total = e.sum(dim=1)
        s["stats"][lo:lo + 512, 0], s["stats"][lo:lo + 512, 1] = high, total
        s["stats"][lo:lo + 512, 2] = total.log() - torch.where(e > 0, e * x, 0.0).sum(dim=1) / total
        del z, x, e
    s["logp_weights"] = up * normal(rows) / rows       # what each text's reward was worth, and a little for staying undecided
    s["entropy_weights"] = torch.full((rows,), up * 0.05 / rows, device="cuda")
    s["grad"] = torch.empty_like(s["z"])
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
        return _own(s, c, _context())
    return {"norm": _norm, "act": _act, "weight": _weight, "score": _score}[c["kind"]](s, c)


def _own(s, c, ctx):
    if c["kind"] == "norm":
        if not c["grad"]:
            ctx.he_layernorm(s["x"], s["y"], EPS, weight=s["weight"], bias=s["bias"], residual=s["residual"], sum_out=s["sum"], stats=s["stats"])
            return {"y": s["y"], "sum": s["sum"]}
        ctx.he_layernorm_grad(s["h"], s["stats"], s["dy"], s["dx"], weight=s["weight"], dsum=s["dsum"], dweight=s["dweight"], dbias=s["dbias"])
        return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    if c["kind"] == "act":
        if not c["grad"]:
            ctx.he_poly_q8(s["u"], s["codes"], s["exponents"], coefs=s["coefs"], y=s["y"])
            return {"y": s["y"], "codes": s["codes"], "exponents": s["exponents"]}
        ctx.he_poly_grad_q8(s["codes"], s["exponents"], s["coefs"], s["dy"], s["du"], dcoefs=s["dcoefs"])
        return {"du": s["du"], "dcoefs": s["dcoefs"]}
    if c["kind"] == "weight":
        ctx.he_weight_grad_q8(s["dy"], s["codes"], s["exponents"], s["dw"])
        return {"dw": s["dw"]}
    if not c["grad"]:
        ctx.he_token_logprobs(s["z"], c["tau"], tokens=s["tokens"], logp=s["logp"], entropy=s["entropy"], values=s["values"], index=s["index"], stats=s["stats"])
        return {"logp": s["logp"], "entropy": s["entropy"], "values": s["values"], "index": s["index"]}
    ctx.he_token_logprobs_grad(s["z"], c["tau"], s["stats"], s["grad"], tokens=s["tokens"], logp_weights=s["logp_weights"], entropy_weights=s["entropy_weights"])
    return {"grad": s["grad"]}


def _norm(s, c):
    t = DTYPES[c["dtype"]]
    w, b = s["weight"].float(), s["bias"].float()
    if not c["grad"]:
        total = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(t)
        h = total.float()
        d = h - h.mean(dim=1, keepdim=True)
        y = d * torch.rsqrt((d * d).mean(dim=1, keepdim=True) + EPS) * w + b
        return {"y": y.to(t), "sum": None if s["residual"] is None else total}
    mean, low, r, _ = s["stats"].split(1, dim=1)
    x, dy = (s["h"].float() - mean - low) * r, s["dy"].float()
    g = dy * w
    dx = r * (g - g.mean(dim=1, keepdim=True) - x * (g * x).mean(dim=1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    p = DTYPES[c["params"]]
    return {"dx": dx.to(t), "dweight": (dy * x).sum(dim=0).to(p), "dbias": dy.sum(dim=0).to(p)}


def _polynomial(u, coefs):
    y = coefs[-1].expand_as(u)
    for a in reversed(coefs[:-1].unbind()):
        y = torch.addcmul(a, y, u)
    return y


def _act(s, c):
    t, coefs = DTYPES[c["dtype"]], s["coefs"]
    if not c["grad"]:
        u = s["u"].float()
        codes, exponents = _kept(u)
        return {"y": _polynomial(u, coefs).to(t), "codes": codes, "exponents": exponents}
    u, dy = _values(s["codes"], s["exponents"]), s["dy"].float()
    slope = coefs[1:] * torch.arange(1, len(coefs), device=u.device)
    sums, power = [], dy
    for _ in coefs.unbind():
        sums.append(power.sum(dtype=torch.float64))
        power = power * u
    return {"du": (dy * _polynomial(u, slope)).to(t), "dcoefs": torch.stack(sums).float()}


def _weight(s, c):
    return {"dw": torch.matmul(s["dy"].float().t(), _values(s["codes"], s["exponents"])).to(DTYPES[c["out"]])}


def _score(s, c):
    tau, tokens = c["tau"], s["tokens"].long()
    z = s["z"].float()
    there = tokens >= 0
    if c["grad"]:
        high, total, entropy, _ = s["stats"].split(1, dim=1)
        x = (z - high) / tau - total.log()
        p = x.exp()
        grad = -p * s["logp_weights"][:, None] * there[:, None] - s["entropy_weights"][:, None] * torch.where(p > 0, p * (x + entropy), 0.0)
        grad.scatter_add_(1, tokens.clamp_min(0)[:, None], (s["logp_weights"] * there)[:, None])
        return {"grad": (grad / tau).to(s["z"].dtype)}
    bits = (z + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7fffffff) - 1, bits)       # in the order of the numbers
    key = (key << 32) + (c["vocab"] - 1 - torch.arange(c["vocab"], device=z.device))      # the lowest index first among equals
    index = (c["vocab"] - 1) - (key.topk(c["k"], dim=1).values & 0xffffffff)
    del key, bits
    high = z.amax(dim=1, keepdim=True)
    x = (z - high) / tau
    e = x.exp()
    total = e.sum(dim=1, keepdim=True)
    entropy = total.log() - torch.where(e > 0, e * x, 0.0).sum(dim=1, keepdim=True) / total
    logp = x.gather(1, tokens.clamp_min(0)[:, None]) - total.log()
    return {"logp": torch.where(there, logp[:, 0], 0.0), "entropy": entropy[:, 0], "values": x.gather(1, index) - total.log(), "index": index.to(torch.int32)}


# ---- from the definitions, in 64 bits

def exact(case, seed):
    c, s = case, prepare(case, seed)
    return {"norm": _exact_norm, "act": _exact_act, "weight": _exact_weight, "score": _exact_score}[c["kind"]](s, c)


def _exact_norm(s, c):
    w, b, dim = s["weight"].double(), s["bias"].double(), c["dim"]
    if not c["grad"]:
        out = {"y": [], "sum": []}
        for lo in range(0, c["rows"], 4096):
            h = s["x"][lo:lo + 4096].double()
            if s["residual"] is not None:
                out["sum"].append(h + s["residual"][lo:lo + 4096].double())
                h = out["sum"][-1].to(DTYPES[c["dtype"]]).double()              # the norm is one of the sum as it is kept
            h = h - (h.sum(1) / dim)[:, None]
            out["y"].append(h / torch.sqrt((h ** 2).sum(1) / dim + EPS)[:, None] * w + b)
        return {"y": torch.cat(out["y"]), "sum": torch.cat(out["sum"]) if out["sum"] else None}
    dx, dw, db = [], torch.zeros_like(w), torch.zeros_like(b)
    for lo in range(0, c["rows"], 4096):
        h, dy = s["h"][lo:lo + 4096].double(), s["dy"][lo:lo + 4096].double()
        h = h - (h.sum(1) / dim)[:, None]
        sigma = torch.sqrt((h ** 2).sum(1) / dim + EPS)[:, None]
        n, g = h / sigma, dy * w
        dw += (dy * n).sum(0)
        db += dy.sum(0)
        d = (g - (g.sum(1) / dim)[:, None] - n * ((g * n).sum(1) / dim)[:, None]) / sigma
        dx.append(d if s["dsum"] is None else d + s["dsum"][lo:lo + 4096].double())
    return {"dx": torch.cat(dx), "dweight": dw, "dbias": db}


def _exact_values(s, lo, hi):
    codes, power = s["codes"][lo:hi].double(), torch.pow(2.0, s["exponents"][lo:hi].double() - 127)
    return codes * power.repeat_interleave(BLOCK, dim=1)[:, :codes.shape[1]]


def _exact_act(s, c):
    a, step = [float(v) for v in s["coefs"]], 2048
    if not c["grad"]:
        out = {"y": [], "codes": [], "exponents": []}
        for lo in range(0, c["rows"], step):
            u = s["u"][lo:lo + step].double()
            out["y"].append(sum(v * u ** i for i, v in enumerate(a)))
            most = torch.stack([p.abs().max(dim=1).values for p in u.split(BLOCK, dim=1)], dim=1)
            e = torch.full_like(most, LEAST)
            while bool((most > F8_MAX * torch.pow(2.0, e)).any()):
                e += (most > F8_MAX * torch.pow(2.0, e)).double()
            out["codes"].append((u / torch.pow(2.0, e).repeat_interleave(BLOCK, dim=1)[:, :c["dim"]]).to(F8).double())
            out["exponents"].append((e + 127).to(torch.uint8))
        return {k: torch.cat(v) for k, v in out.items()}
    du, dc = [], torch.zeros(len(a), dtype=torch.float64, device="cuda")
    for lo in range(0, c["rows"], step):
        u, dy = _exact_values(s, lo, lo + step), s["dy"][lo:lo + step].double()
        du.append(dy * sum(i * v * u ** (i - 1) for i, v in enumerate(a) if i))
        dc += torch.stack([(dy * u ** i).sum() for i in range(len(a))])
    return {"du": torch.cat(du), "dcoefs": dc}


def _exact_weight(s, c):
    dw = torch.zeros((c["n"], c["k"]), dtype=torch.float64, device="cuda")
    for lo in range(0, c["m"], 4096):
        dw += s["dy"][lo:lo + 4096].double().t() @ _exact_values(s, lo, lo + 4096)
    return {"dw": dw}


def _exact_score(s, c):
    out = {"grad": []} if c["grad"] else {"logp": [], "entropy": [], "values": [], "index": []}
    for lo in range(0, c["rows"], 128):
        cut = slice(lo, lo + 128)
        z, y = s["z"][cut].double(), s["tokens"][cut].long()
        logp = torch.log_softmax(z / c["tau"], dim=1)
        p = torch.softmax(z / c["tau"], dim=1)
        entropy = -torch.xlogy(p, p).sum(dim=1)
        if c["grad"]:
            hot = torch.zeros_like(z).scatter_(1, y.clamp_min(0)[:, None], 1.0)
            a = torch.where(y >= 0, s["logp_weights"][cut].double(), 0.0)[:, None]
            out["grad"].append((a * (hot - p) - s["entropy_weights"][cut].double()[:, None] * (torch.xlogy(p, p) + p * entropy[:, None])) / c["tau"])
        else:
            index = z.sort(dim=1, descending=True, stable=True).indices[:, :c["k"]]
            out["logp"].append(torch.where(y >= 0, logp.gather(1, y.clamp_min(0)[:, None])[:, 0], 0.0))
            out["entropy"].append(entropy)
            out["values"].append(logp.gather(1, index))
            out["index"].append(index.to(torch.int32))
    return {k: torch.cat(v) for k, v in out.items()}
