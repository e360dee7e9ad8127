"""Timed operators of the update phase: the product with a layer's weights and
its epilogue, the class loss, the optimizer step.

* ``linear``  Y = act(alpha X W + b + beta R), and with ``train`` its gradients
* ``loss``    softmax cross entropy of the logits X W + b against one class a
              row, rows of target -100 left out; with ``train`` the gradients
              of X, W and b for an upstream gradient (a loss scale)
* ``adamw``   one AdamW step over a list of tensors, both moments held in 32
              bits or in blocks of 256 8-bit codes

The plain forms compute in 32 bits and round once at the end. Masks of a ReLU
are taken from 64-bit sums, since a sum next to zero may change sides.
"""
from __future__ import annotations

import math

import torch

own = False

IGNORE = -100
BLOCK = 256
LR, BETAS, EPS, DECAY = 1e-3, (0.9, 0.999), 1e-8, 0.01
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one token through a square layer, weights stored output-major: the
        # smallest product, bound by reading the weights
        {"name": "linear_token", "kind": "linear", "dtype": "bf16", "n": 1, "k": 4096, "m": 4096, "act": "silu",
         "bias": True, "residual": False, "out_major": True, "train": False},
        # a Yelp-shaped graph's first layer, 300 features to 512 hidden units,
        # every node a row, in single precision as the aggregation takes it
        {"name": "linear_nodes", "kind": "linear", "dtype": "fp32", "n": 716847, "k": 300, "m": 512, "act": "relu",
         "bias": True, "residual": False, "out_major": False, "train": False},
        # a Reddit-shaped graph's first layer in training: 602 features, 256
        # hidden units, with its gradients (the weights' sum runs over nodes)
        {"name": "linear_nodes_train", "kind": "linear", "dtype": "fp32", "n": 232965, "k": 602, "m": 256,
         "act": "gelu", "bias": True, "residual": False, "out_major": False, "train": True},
        # odd sizes everywhere, half precision, residual inside the ReLU
        {"name": "linear_ragged_train", "kind": "linear", "dtype": "fp16", "n": 5003, "k": 1021, "m": 2045,
         "act": "relu", "bias": True, "residual": True, "out_major": False, "train": True},
        # a block's second projection over a batch of tokens, with the
        # residual stream added, forward and gradients
        {"name": "linear_tokens_train", "kind": "linear", "dtype": "bf16", "n": 16384, "k": 8192, "m": 4096,
         "act": "none", "bias": False, "residual": True, "out_major": True, "train": True},
        # a small evaluation batch: ragged rows, a thousand classes
        {"name": "loss_eval", "kind": "loss", "dtype": "bf16", "n": 333, "k": 512, "v": 1000, "valid": 1.0,
         "bias": True, "out_major": True, "train": False},
        # Reddit-shaped node classification: 41 classes, two thirds labelled
        {"name": "loss_nodes_train", "kind": "loss", "dtype": "fp32", "n": 232965, "k": 256, "v": 41, "valid": 0.66,
         "bias": True, "out_major": False, "train": True},
        # half precision with odd sizes and a mid-size vocabulary
        {"name": "loss_ragged_train", "kind": "loss", "dtype": "fp16", "n": 3001, "k": 1000, "v": 50021, "valid": 0.9,
         "bias": True, "out_major": True, "train": True},
        # a large vocabulary over a batch of tokens
        {"name": "loss_tokens_train", "kind": "loss", "dtype": "bf16", "n": 8192, "k": 4096, "v": 131072, "valid": 0.97,
         "bias": False, "out_major": True, "train": True},
        # the two weight matrices of a 300-512-100 network
        {"name": "adamw_gcn", "kind": "adamw", "dtype": "fp32", "bits": 32, "tensors": 2, "largest": 512 * 300,
         "smallest": 512 * 100},
        # many tensors of a mid-size network, from vectors to matrices, 32-bit
        # states beside 16-bit parameters with 32-bit masters
        {"name": "adamw_many", "kind": "adamw", "dtype": "bf16", "bits": 32, "tensors": 290, "largest": 4096 * 4096,
         "smallest": 37},
        # a large network's shard with 8-bit states
        {"name": "adamw_8bit", "kind": "adamw", "dtype": "fp32", "bits": 8, "tensors": 120, "largest": 4096 * 8192,
         "smallest": 1000},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "loss", "loss", "adamw"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    if kind == "adamw":
        tensors = _log(rng, 1, 300)
        largest = _log(rng, 1000, min(4096 * 8192, 300_000_000 // tensors + 1000))
        return {"kind": kind, "dtype": dtype, "bits": rng.choice([8, 32]), "tensors": tensors, "largest": largest,
                "smallest": _log(rng, 1, largest)}
    case = {"kind": kind, "dtype": dtype, "n": _log(rng, 1, 700000), "k": _log(rng, 16, 8192)}
    case["train"] = rng.random() < 0.6
    case["bias"] = rng.random() < 0.6
    case["out_major"] = rng.random() < 0.5
    if kind == "linear":
        case["m"] = _log(rng, 16, 16384)
        # a ReLU's gradient in single precision hangs on the sign of sums next to zero
        acts = ["none", "gelu", "silu"] + (["relu"] if dtype != "fp32" or not case["train"] else [])
        case["act"] = rng.choice(acts)
        case["residual"] = rng.random() < 0.5
        out = "m"
    else:
        case["v"] = _log(rng, 2, 131072)
        case["valid"] = rng.choice([1.0, 0.9, 0.5, 0.08])
        out = "v"
    # at most the work, and the values, of the largest listed case
    most_work, most_values = (2.0e12, 6e8)
    for _ in range(64):
        n, k, m = case["n"], case["k"], case[out]
        if 2.0 * n * k * m <= most_work and n * k + n * m + k * m <= most_values:
            break
        case["n"] = max(1, n * 2 // 3)
        case["k"] = max(16, k * 5 // 6)
    return case


# ------------------------------------------------------------------ inputs
def _generator(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed * 2654435761 % (1 << 62) + 29)
    return g


def _normal(rows, cols, dtype, g, scale=1.0):
    """N(0, scale^2), rows a whole number of 16 bytes apart, as the library's
    dense matrices are."""
    unit = 16 // dtype.itemsize
    ld = (cols + unit - 1) // unit * unit
    t = torch.empty((rows, ld), dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // ld)
    for i in range(0, rows, step):
        part = t[i:i + step]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * scale)
    return t[:, :cols]


def _weight(k, m, out_major, dtype, g, scale):
    return _normal(m, k, dtype, g, scale).t() if out_major else _normal(k, m, dtype, g, scale)


def _shapes(case):
    """Element counts from the largest to the smallest, evenly over the
    logarithm, most of them not whole blocks."""
    t, hi, lo = case["tensors"], math.log(case["largest"]), math.log(case["smallest"])
    return [int(round(math.exp(hi + (lo - hi) * j / max(1, t - 1)))) for j in range(t)]


def _pieces(flat, shapes, unit=1):
    """Views of one buffer, each tensor starting at a whole block."""
    got, at = [], 0
    for n in shapes:
        blocks = (n + BLOCK - 1) // BLOCK
        got.append(flat[at:at + (n if unit == 1 else blocks)])
        at += blocks * BLOCK // unit
    return got


def _optimizer_state(case, seed, g, dtype):
    """Parameters, gradients and moments as a run leaves them, each kind in one
    buffer that the tensors are views of."""
    shapes = _shapes(case)
    blocks = sum((n + BLOCK - 1) // BLOCK for n in shapes)
    total = blocks * BLOCK

    def filled(make, to):
        t = torch.empty(total, dtype=to, device="cuda")
        for i in range(0, total, 1 << 26):
            part = t[i:i + (1 << 26)]
            part.copy_(make(part.numel()))
        return t

    def normal(scale):
        return lambda n: torch.randn(n, generator=g, device="cuda") * scale

    def uniform(n):
        return torch.rand(n, generator=g, device="cuda")

    flat = {"grads": filled(normal(1e-3), dtype)}
    if dtype != torch.float32:
        flat["masters"] = filled(normal(0.02), torch.float32)
        flat["params"] = flat["masters"].to(dtype)
    else:
        flat["params"] = filled(normal(0.02), torch.float32)
    if case["bits"] == 8:
        flat["m"] = filled(lambda n: (uniform(n) * 254 - 127).round_(), torch.int8)
        flat["v"] = filled(lambda n: (uniform(n) * 254 + 1).round_(), torch.uint8)
        flat["ms"] = uniform(blocks) * 1e-3 + 1e-4
        flat["vs"] = uniform(blocks) * 2e-3 + 1e-3
        flat["m_out"], flat["v_out"] = (torch.zeros(total, dtype=torch.float32, device="cuda") for _ in range(2))
    else:
        flat["m"] = filled(normal(3e-4), torch.float32)
        flat["v"] = filled(lambda n: uniform(n) ** 2 * 1e-6 + 1e-12, torch.float32)
    at = 0
    for n in shapes:  # what lies between two tensors is zero, which a step leaves as it is
        end = at + (n + BLOCK - 1) // BLOCK * BLOCK
        if at + n < end:
            for name, t in flat.items():
                if name not in ("ms", "vs"):
                    t[at + n:end].zero_()
        at = end
    s = {name: _pieces(t, shapes, BLOCK if name in ("ms", "vs") else 1) for name, t in flat.items()}
    s.update(flat=flat, step=torch.full((1,), 100 + seed % 7, dtype=torch.int64, device="cuda"), at=100 + seed % 7,
             seed=seed)
    return s


def prepare(case, seed):
    g = _generator(seed)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    s = {"case": dict(case)}
    if kind == "adamw":
        s.update(_optimizer_state(case, seed, g, dtype))
        return s
    n, k = case["n"], case["k"]
    out = case["m"] if kind == "linear" else case["v"]
    s["x"] = _normal(n, k, dtype, g)
    s["w"] = _weight(k, out, case["out_major"], dtype, g, (1.0 if kind == "linear" else 2.0) / math.sqrt(k))
    s["b"] = (torch.randn(out, generator=g, device="cuda") * 0.1).to(dtype) if case["bias"] else None
    if kind == "linear":
        s["r"] = _normal(n, out, dtype, g) if case["residual"] else None
        s["dy"] = _normal(n, out, dtype, g) if case["train"] else None
        s["alpha"], s["beta"] = 1.0, (0.5 if case["residual"] else 1.0)
    else:
        # classes as words are: a few frequent ones, a long tail
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        t = (torch.exp(u * math.log(out + 1.0)) - 1.0).long().clamp_(0, out - 1)
        t[torch.rand(n, generator=g, device="cuda") >= case["valid"]] = IGNORE
        s["t"] = t
        s["upstream"] = torch.full((), 1024.0 if dtype == torch.float16 else 1.0, device="cuda")
    if case["train"]:
        for name in ("x", "w", "b", "r"):
            if s.get(name) is not None:
                s[name].requires_grad_()
    return s


# --------------------------------------------------------------- plain forms
def _act(z, act):
    """act(z) and its derivative."""
    if act == "relu":
        return torch.clamp_min(z, 0), (z > 0).to(z.dtype)
    if act == "gelu":
        phi = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return z * p, p * (1 + z * (1 - p))
    return z, None


def _linear_plain(s, t=torch.float32):
    case = s["case"]
    x, w, b, r = (None if s[name] is None else s[name].detach().to(t) for name in ("x", "w", "b", "r"))
    dtype, act = s["x"].dtype, case["act"]
    at = torch.float64 if case["train"] and act == "relu" else t
    z = (x.to(at) @ w.to(at)) * s["alpha"]
    if b is not None:
        z = z + b
    if r is not None:
        z = z + s["beta"] * r
    y, slope = _act(z, act)
    y, slope = y.to(t), None if slope is None or not case["train"] else slope.to(t)
    del z
    last = (lambda v: v) if t == torch.float64 else (lambda v: v.to(dtype))
    if not case["train"]:
        return last(y)
    dz = s["dy"].to(t)
    dz = dz if slope is None else dz * slope
    got = {"y": last(y), "dx": last((dz @ w.t()) * s["alpha"]), "dw": last((x.t() @ dz) * s["alpha"])}
    if b is not None:
        got["db"] = last(dz.sum(0, dtype=torch.float64).to(t))
    if r is not None:
        got["dr"] = last(s["beta"] * dz)
    return got


def _loss_plain(s, t=torch.float32):
    case, dtype = s["case"], s["x"].dtype
    x, w = s["x"].detach().to(t), s["w"].detach().to(t)
    target = s["t"]
    valid = target != IGNORE
    count = valid.sum()
    logits = x @ w
    if s["b"] is not None:
        logits += s["b"].detach().to(t)
    top = logits.amax(1, keepdim=True)
    at = logits.gather(1, target.clamp_min(0)[:, None])
    logits.sub_(top).exp_()
    total = logits.sum(1, keepdim=True)
    rows = torch.log(total) + top - at
    rows = torch.where(valid[:, None], rows, torch.zeros_like(rows))
    loss = (rows.double().sum() / count.clamp_min(1)).to(t)
    if not case["train"]:
        return loss
    last = (lambda v: v) if t == torch.float64 else (lambda v: v.to(dtype))
    g = (valid.to(t) * (s["upstream"].to(t) / count.clamp_min(1).to(t)))[:, None]
    logits.div_(total)
    logits.scatter_add_(1, target.clamp_min(0)[:, None], -torch.ones_like(g))
    logits.mul_(g)
    got = {"loss": loss, "dx": last(logits @ w.t()), "dw": last(x.t() @ logits)}
    if s["b"] is not None:
        got["db"] = last(logits.sum(0, dtype=torch.float64).to(t))
    return got


_M64 = (1 << 64) - 1


def _signed(v):
    v &= _M64
    return v - (1 << 64) if v >> 63 else v


def _bits(seed, step, n):
    """SplitMix64 (Steele, Lea and Flood 2014) seeded with `seed`, output
    number step 2^40 + i + 1 for element i (each tensor's first one at a whole
    block behind the tensor before); 64-bit words that wrap."""
    z = torch.arange(n, dtype=torch.int64, device="cuda") + (step * (1 << 40) + 1)
    z = z * _signed(0x9E3779B97F4A7C15) + _signed(seed)
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _blocks(x):
    """The largest value of each block of a non-negative vector."""
    return x.view(-1, BLOCK).amax(1)


def _spread(scale, n):
    return scale[:, None].expand(-1, BLOCK).reshape(n)


def _encode(x, levels, u):
    """Codes of a non-negative vector: the square root of its share of the
    block's largest, times `levels`, rounded up with that chance."""
    scale = _blocks(x)
    share = _spread(torch.where(scale > 0, scale, torch.ones_like(scale)), x.numel())
    return torch.floor(torch.sqrt(x / share) * levels + u).clamp_max(levels), scale


def _adamw_plain(s):
    """All tensors at once, every operation a rounding of its own to 32 bits, in
    the order that defines the step (codes next to a border hang on it)."""
    flat, code = s["flat"], s["case"]["bits"] == 8
    s["step"] += 1
    s["at"] += 1
    step, n = s["at"], flat["grads"].numel()
    b1, b2, c1, c2 = (_f32(v) for v in (BETAS[0], BETAS[1], 1 - BETAS[0], 1 - BETAS[1]))
    rate, unbias = _f32(LR / (1 - BETAS[0] ** step)), _f32(1 / math.sqrt(1 - BETAS[1] ** step))
    keep, eps = _f32(1 - LR * DECAY), _f32(EPS)
    g = flat["grads"].float()
    if code:
        m = _decode(flat["m"], 127) * _spread(flat["ms"], n)
        r = _decode(flat["v"], 255) * _spread(flat["vs"], n)
        v = r * r
    else:
        m, v = flat["m"], flat["v"]
    m = m * b1 + g * c1
    v = v * b2 + (g * c2) * g
    r = torch.sqrt(v)
    p = flat["masters" if "masters" in flat else "params"]
    p.copy_(p * keep - (m * rate) / (r * unbias + eps))
    if "masters" in flat:
        flat["params"].copy_(p)
    if code:
        z = _bits(s["seed"], step, n)
        q, scale = _encode(m.abs(), 127.0, (z & 0xFFFFFF).float() * 2.0 ** -24)
        flat["m"].copy_(torch.where(m < 0, -q, q))
        flat["ms"].copy_(scale)
        flat["m_out"].copy_(_decode(flat["m"], 127) * _spread(scale, n))
        q, scale = _encode(r, 255.0, ((z >> 24) & 0xFFFFFF).float() * 2.0 ** -24)
        flat["v"].copy_(torch.where(r > 0, q.clamp_min(1.0), q))
        flat["vs"].copy_(scale)
        r = _decode(flat["v"], 255) * _spread(scale, n)
        flat["v_out"].copy_(r * r)
    else:
        flat["m"].copy_(m)
        flat["v"].copy_(v)


def _f32(v):
    return float(torch.tensor(v, dtype=torch.float32))


def _decode(code, levels):
    w = code.float() * _f32(1 / levels)
    return w * w.abs()


def _state(s):
    """The buffers after the step: parameters (and masters), both moments, from
    codes the values that they stand for."""
    flat = s["flat"]
    got = {name: flat[name] for name in ("params", "masters") if name in flat}
    code = "m_out" in flat
    return {**got, "m": flat["m_out" if code else "m"], "v": flat["v_out" if code else "v"]}


# ----------------------------------------------------------------------- run
def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        import paper_2210_10737_amd as rsc
        if kind == "linear":
            y = rsc.linear(s["x"], s["w"], s["b"], residual=s["r"], act=case["act"], alpha=s["alpha"], beta=s["beta"])
            if not case["train"]:
                return y
            wanted = {"dx": s["x"], "dw": s["w"], "db": s["b"], "dr": s["r"]}
            wanted = {name: t for name, t in wanted.items() if t is not None}
            return {"y": y.detach(), **dict(zip(wanted, torch.autograd.grad(y, list(wanted.values()), s["dy"])))}
        if kind == "loss":
            loss = rsc.linear_cross_entropy(s["x"], s["w"], s["t"], s["b"], ignore_index=IGNORE)
            if not case["train"]:
                return loss
            wanted = {"dx": s["x"], "dw": s["w"], "db": s["b"]}
            wanted = {name: t for name, t in wanted.items() if t is not None}
            return {"loss": loss.detach(),
                    **dict(zip(wanted, torch.autograd.grad(loss, list(wanted.values()), s["upstream"])))}
        rsc.adamw_step(s["params"], s["grads"], s["m"], s["v"], s["step"], lr=LR, betas=BETAS, eps=EPS,
                       weight_decay=DECAY, masters=s.get("masters"), exp_avg_scales=s.get("ms"),
                       exp_avg_sq_scales=s.get("vs"), seed=s["seed"])
        if case["bits"] == 8:
            rsc.adamw_moments(s["m"], s["v"], s["ms"], s["vs"], out=(s["m_out"], s["v_out"]))
        return _state(s)
    if kind == "linear":
        return _linear_plain(s)
    if kind == "loss":
        return _loss_plain(s)
    _adamw_plain(s)
    return _state(s)


# -------------------------------------------------------------- the floor
def work(case):
    """Each input read once, each output written once; two operations per
    product and sum of the matrix products, the gradients' among them."""
    size = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "adamw":
        n = sum(_shapes(case))
        # moments in and out; from codes, their values out too
        state = 2 * 8 if case["bits"] == 32 else 2 * 2 + 4 * 4 / BLOCK + 8
        return {"bytes": n * (3 * size + state + (8 if size == 2 else 0)), "flops": 15.0 * n}
    n, k = case["n"], case["k"]
    if case["kind"] == "linear":
        m = case["m"]
        values = n * k + k * m + n * m * (2 if case["residual"] else 1) + (m if case["bias"] else 0)
        if case["train"]:
            # dy in; dx, dw, db, dr out
            values += n * m + values - n * m
        return {"bytes": float(size) * values, "flops": (6.0 if case["train"] else 2.0) * n * k * m}
    v = case["v"]
    values = n * k + k * v + (v if case["bias"] else 0)
    rows = n * case["valid"]
    return {"bytes": float(size) * values * (2 if case["train"] else 1) + 8.0 * n,
            "flops": (6.0 if case["train"] else 2.0) * rows * k * v}


# ------------------------------------------------------------- 64-bit truth
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(case, s)
    x, w = s["x"].detach().double(), s["w"].detach().double()
    b = None if s["b"] is None else s["b"].detach().double()
    if case["kind"] == "linear":
        z = s["alpha"] * torch.matmul(x, w)
        z = z if b is None else z + b
        z = z if s["r"] is None else z + s["beta"] * s["r"].detach().double()
        act = case["act"]
        if act == "none":
            y, slope = z, torch.ones_like(z)
        elif act == "relu":
            y, slope = torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0)
        elif act == "gelu":
            cdf = torch.erfc(-z / math.sqrt(2.0)) / 2
            y, slope = z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        else:
            sig = torch.sigmoid(z)
            y, slope = z * sig, sig + z * sig * (1 - sig)
        if not case["train"]:
            return y
        dz = slope * s["dy"].double()
        got = {"y": y, "dx": s["alpha"] * torch.matmul(dz, w.t()), "dw": s["alpha"] * torch.matmul(x.t(), dz)}
        if b is not None:
            got["db"] = dz.sum(0)
        if s["r"] is not None:
            got["dr"] = s["beta"] * dz
        return got
    keep = (s["t"] != IGNORE).nonzero()[:, 0]
    target, n = s["t"][keep], max(1, keep.numel())
    xs = x[keep]
    logits = torch.matmul(xs, w)
    logits = logits if b is None else logits + b
    lse = torch.logsumexp(logits, 1)
    loss = (lse - logits[torch.arange(keep.numel(), device="cuda"), target]).sum() / n
    if not case["train"]:
        return loss
    p = logits.sub_(lse[:, None]).exp_()
    p[torch.arange(keep.numel(), device="cuda"), target] -= 1.0
    p *= float(s["upstream"]) / n
    dx = torch.zeros_like(x)
    dx[keep] = torch.matmul(p, w.t())
    got = {"loss": loss, "dx": dx, "dw": torch.matmul(xs.t(), p)}
    if b is not None:
        got["db"] = p.sum(0)
    return got


def _exact_adamw(case, s):
    """The moments of 8 bits hang on the draws: their values are left out."""
    step = s["at"] + 1
    flat, code = s["flat"], case["bits"] == 8
    p = torch.zeros_like(flat["params"], dtype=torch.float64)
    p.copy_(flat["masters" if "masters" in flat else "params"])
    moments = [torch.zeros_like(p), torch.zeros_like(p)]
    if not code:
        moments[0].copy_(flat["m"])
        moments[1].copy_(flat["v"])
    shapes = _shapes(case)
    for j, (x, m, v) in enumerate(zip(_pieces(p, shapes), *(_pieces(t, shapes) for t in moments))):
        g = s["grads"][j].double()
        if code:
            block = torch.arange(g.numel(), device="cuda") // BLOCK
            q, r = s["m"][j].double() / 127, s["v"][j].double() / 255
            m.copy_(q * q.abs() * s["ms"][j].double()[block])
            v.copy_((r * r * s["vs"][j].double()[block]) ** 2)
        m.mul_(BETAS[0]).add_(g, alpha=1 - BETAS[0])
        v.mul_(BETAS[1]).add_(g * g, alpha=1 - BETAS[1])
        root = torch.sqrt(v / (1 - BETAS[1] ** step))
        x.copy_(x * (1 - LR * DECAY) - LR * (m / (1 - BETAS[0] ** step)) / (root + EPS))
    got = {"params": p, "m": None if code else moments[0], "v": None if code else moments[1]}
    return {**got, "masters": p} if "masters" in flat else got
