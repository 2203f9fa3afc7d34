"""Performance cases of a layer with its activation and residual, and of what a vocabulary's logits are for.

Three kinds of work, each in its plain form and through the public entry points of paper_1712_04432_amd:

* ``linear``    a fully connected layer's product with bias, activation and residual in its epilogue, and the products
                of its backward pass with the derivative of the activation below and the residual's gradient in theirs;
* ``distill``   the divergence of a student's softmax from a teacher of which only the top logits are known, and its
                gradient by the student's logits;
* ``logprobs``  the log probabilities of given tokens, with the entropy and the top alternatives, and in training the
                gradient of the first two.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"


# ------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # Eight single tokens through a layer that ends a residual block: the weights stream once.
        {"name": "linear_decode", "kind": "linear", "pass": "fwd", "dtype": "bf16", "B": 8, "d_in": 4096, "d_out": 4096,
         "act": "none", "bias": True, "residual": True, "keep": False},
        # A serving batch through the layer that widens: still weights, but 64 rows of products for each.
        {"name": "linear_serve", "kind": "linear", "pass": "fwd", "dtype": "bf16", "B": 64, "d_in": 4096, "d_out": 16384,
         "act": "silu", "bias": True, "residual": False, "keep": False},
        # The same layer in training, the sums before the activation kept for its backward pass.
        {"name": "linear_fwd_large", "kind": "linear", "pass": "fwd", "dtype": "bf16", "B": 8192, "d_in": 4096,
         "d_out": 16384, "act": "gelu_tanh", "bias": True, "residual": False, "keep": True},
        # The backward products of the layer that narrows again: the gradient before the activation below, the
        # weights' and the bias's. The largest case.
        {"name": "linear_bwd_large", "kind": "linear", "pass": "bwd", "dtype": "bf16", "B": 8192, "d_in": 16384,
         "d_out": 4096, "act": "gelu_tanh", "bias": True, "residual": False, "keep": False},
        # Single precision on widths that are no multiple of anything, all passes, a residual in both.
        {"name": "linear_f32_odd", "kind": "linear", "pass": "both", "dtype": "f32", "B": 1000, "d_in": 1023,
         "d_out": 517, "act": "gelu", "bias": True, "residual": True, "keep": True},
        # The smallest: the thousand classes of the framework's own networks, latency.
        {"name": "distill_classes", "kind": "distill", "dtype": "f32", "B": 64, "V": 1000, "K": 8, "temperature": 1.0,
         "mass": False, "pad": 0, "grad": True},
        # A training step's tokens over a large vocabulary, a sixteenth of them padding: read once, written once.
        {"name": "distill_large", "kind": "distill", "dtype": "bf16", "B": 4096, "V": 131072, "K": 64,
         "temperature": 2.0, "mass": False, "pad": 256, "grad": True},
        # Single precision, an odd vocabulary, and a teacher whose top logits come with their true probabilities.
        {"name": "distill_f32_odd", "kind": "distill", "dtype": "f32", "B": 500, "V": 50021, "K": 20,
         "temperature": 1.0, "mass": True, "pad": 0, "grad": True},
        # A decoding step that reports twenty alternatives of each token: few long rows.
        {"name": "logprobs_decode", "kind": "logprobs", "dtype": "bf16", "B": 16, "V": 131072, "top": 20,
         "temperature": 1.0, "pad": 0, "bwd": False},
        # Scoring prompts, five alternatives each.
        {"name": "logprobs_score", "kind": "logprobs", "dtype": "bf16", "B": 2048, "V": 131072, "top": 5,
         "temperature": 1.0, "pad": 0, "bwd": False},
        # A policy's training step: log probability and entropy of each token, and their gradient.
        {"name": "logprobs_train", "kind": "logprobs", "dtype": "bf16", "B": 8192, "V": 32768, "top": 0,
         "temperature": 1.0, "pad": 512, "bwd": True},
        # Single precision, an odd vocabulary, a temperature.
        {"name": "logprobs_f32_odd", "kind": "logprobs", "dtype": "f32", "B": 333, "V": 100003, "top": 1,
         "temperature": 0.7, "pad": 0, "bwd": True},
    ]


ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width: most are multiples of 64 or 8 as programs choose them, the others as they come."""
    w, how = _log(rng, lo, hi), rng.random()
    if how < 0.55:
        return max(64, w // 64 * 64)
    return max(8, w // 8 * 8) if how < 0.8 else w


MOST_FLOPS = {"bf16": 2.1e12, "f32": 6.0e10}
MOST_LOGITS = 500_000_000


def draw(rng):
    while True:
        kind = rng.choice(["linear", "linear", "distill", "logprobs"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        if kind == "linear":
            c = {"kind": kind, "pass": rng.choice(["fwd", "fwd", "bwd", "both"]), "dtype": dtype,
                 "B": _log(rng, 1, 16384), "d_in": _width(rng, 64, 16384), "d_out": _width(rng, 64, 16384),
                 "act": rng.choice(ACTS), "bias": rng.random() < 0.7, "residual": rng.random() < 0.5,
                 "keep": rng.random() < 0.5}
            if c["d_in"] * c["d_out"] <= 100_000_000 and work(c)["flops"] <= MOST_FLOPS[dtype]:
                return c
            continue
        B, V = _log(rng, 1, 16384), _width(rng, 500, 160_000)
        c = {"kind": kind, "dtype": dtype, "B": B, "V": V, "temperature": rng.choice([1.0, 1.0, 0.7, 2.0]),
             "pad": rng.choice([0, 0, B // 10])}
        if kind == "distill":
            c.update(K=rng.choice([1, 8, 20, 50, 64, 128]), mass=rng.random() < 0.3, grad=rng.random() < 0.8)
            most = MOST_LOGITS
        else:
            c.update(top=rng.choice([0, 0, 1, 5, 20]), bwd=rng.random() < 0.4)
            most = MOST_LOGITS if c["top"] == 0 else MOST_LOGITS // 4
        if B * V <= most // (2 if dtype == "f32" else 1):
            return c


# ------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape, scale=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale).to(dtype)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _logits(g, case):
    """Logits as a network gives them: a spread of about two, some tokens liked better everywhere, and a few that are
    ruled out."""
    B, V = case["B"], case["V"]
    z = _normal(g, B, V, scale=2.0, dtype=_dtype(case))
    liked = _normal(g, V)
    liked[torch.randint(0, V, (max(1, V // 1000),), generator=g, device=DEV)] = -math.inf
    z += liked.to(z.dtype)
    return z


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    {"linear": _prepare_linear, "distill": _prepare_distill, "logprobs": _prepare_logprobs}[case["kind"]](s, case, g)
    return s


def _workspace(nbytes):
    return torch.zeros(nbytes, dtype=torch.uint8, device=DEV) if nbytes else None


def _prepare_linear(s, c, g):
    B, d_in, d_out, dt = c["B"], c["d_in"], c["d_out"], _dtype(c)
    s["w"] = _normal(g, d_out, d_in, scale=1.0 / math.sqrt(d_in), dtype=dt)
    s["x"] = _normal(g, B, d_in, dtype=dt)
    s["bias"] = _normal(g, d_out, scale=0.1) if c["bias"] else None
    s["residual"] = _normal(g, B, d_out, dtype=dt) if c["residual"] else None
    if c["pass"] != "fwd":
        s["dy"] = _normal(g, B, d_out, scale=0.05, dtype=dt)
        s["z_below"] = _normal(g, B, d_in, dtype=dt) if c["act"] != "none" else None
        s["dresidual"] = _normal(g, B, d_in, scale=0.05, dtype=dt) if c["residual"] else None
    if own:
        import paper_1712_04432_amd as imbd
        if c["pass"] != "bwd":
            s["y"] = torch.zeros(B, d_out, dtype=dt, device=DEV)
            s["z"] = torch.zeros(B, d_out, dtype=dt, device=DEV) if c["keep"] else None
            s["ws_fwd"] = _workspace(imbd.linear_workspace_bytes(0, imbd.dtype_code(dt), d_out, d_in, B))
        if c["pass"] != "fwd":
            s.update(dw=torch.zeros(d_out, d_in, device=DEV), db=torch.zeros(d_out, device=DEV),
                     dx=torch.zeros(B, d_in, dtype=dt, device=DEV))
            s["ws_bwd"] = _workspace(imbd.linear_workspace_bytes(1, imbd.dtype_code(dt), d_out, d_in, B))


def _prepare_distill(s, c, g):
    B, V, K = c["B"], c["V"], c["K"]
    z = _logits(g, c)
    # The teacher's top tokens, K different ones of each row from the most probable on; the student's logits there
    # are near the teacher's. The last quarter is missing in every seventh row.
    step = next(p for p in (7919, 7907, 7901) if V % p)
    first = torch.randint(0, V, (B, 1), generator=g, device=DEV)
    ids = (first + step * torch.arange(K, device=DEV)) % V
    t = 9.0 - 1.5 * torch.log1p(torch.arange(K, device=DEV, dtype=torch.float32)) + _normal(g, B, K, scale=0.05)
    z.scatter_(1, ids, (t + _normal(g, B, K)).to(z.dtype))
    ids[::7, K - K // 4:] = -1
    s["logits"], s["ids"], s["teacher"] = z, ids.to(torch.int32), t
    tau = c["temperature"]
    s["lse"] = torch.logsumexp(t / tau, 1) + 0.05 + _normal(g, B, scale=0.02).abs() if c["mass"] else None
    s["weight"] = torch.ones(B, device=DEV) if c["pad"] else None
    if c["pad"]:
        s["weight"][B - c["pad"]:] = 0.0
    s["inv_batch"] = 1.0 / (B - c["pad"])
    if own:
        import paper_1712_04432_amd as imbd
        s.update(loss=torch.zeros(1, device=DEV), row_loss=torch.zeros(B, device=DEV),
                 dlogits=torch.zeros(B, V, dtype=z.dtype, device=DEV) if c["grad"] else None,
                 ws=_workspace(imbd.distill_workspace_bytes(B, V, K)))


def _prepare_logprobs(s, c, g):
    B, V, n = c["B"], c["V"], c["top"]
    s["logits"] = _logits(g, c)
    # (a sampled token is a likely one: the best of a few)
    some = torch.randint(0, V, (B, 16), generator=g, device=DEV)
    tokens = some.gather(1, s["logits"].gather(1, some).float().argmax(1, keepdim=True)).squeeze(1).to(torch.int32)
    if c["pad"]:
        tokens[B - c["pad"]:] = -1
    s["tokens"] = tokens
    if c["bwd"]:
        s["dlogp"] = _normal(g, B, scale=1.0 / B)
        s["dentropy"] = torch.full((B,), -0.01 / B, device=DEV)
        if c["pad"]:
            s["dentropy"][B - c["pad"]:] = 0.0
    if own:
        import paper_1712_04432_amd as imbd
        s.update(logp=torch.zeros(B, device=DEV), entropy=torch.zeros(B, device=DEV), lse=torch.zeros(B, device=DEV),
                 top_ids=torch.zeros(B, n, dtype=torch.int32, device=DEV) if n else None,
                 top_logp=torch.zeros(B, n, device=DEV) if n else None,
                 dlogits=torch.zeros_like(s["logits"]) if c["bwd"] else None,
                 ws=_workspace(imbd.token_logprobs_workspace_bytes(B, V, n)))


# ------------------------------------------------------------------------------------ one pass
def run(s):
    return {"linear": _linear, "distill": _distill, "logprobs": _logprobs}[s["case"]["kind"]](s)


def _act(name, z):
    if name == "relu":
        return z.clamp(min=0.0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        density = torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * density
    if name == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    p = 1.0 / (1.0 + torch.exp(-z))
    return p * (1.0 + z * (1.0 - p))


def _linear(s):
    c = s["case"]
    out = []
    if own:
        import paper_1712_04432_amd as imbd
        if c["pass"] != "bwd":
            imbd.linear_fwd(s["w"], s["x"], s["y"], bias=s["bias"], act=c["act"], residual=s["residual"], z=s["z"],
                            ws=s["ws_fwd"])
            out += [s["y"]] + ([s["z"]] if c["keep"] else [])
        if c["pass"] != "fwd":
            imbd.linear_bwd(s["w"], s["dy"], s["x"], dw=s["dw"], db=s["db"], dx=s["dx"], act=c["act"],
                            z=s["z_below"], residual=s["dresidual"], ws=s["ws_bwd"])
            out += [s["dw"], s["db"], s["dx"]]
        return out
    dt, w, x = _dtype(c), s["w"].float(), s["x"].float()
    if c["pass"] != "bwd":
        z = torch.matmul(x, w.t())
        if s["bias"] is not None:
            z = z + s["bias"]
        y = _act(c["act"], z)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out += [y.to(dt)] + ([z.to(dt)] if c["keep"] else [])
    if c["pass"] != "fwd":
        dy = s["dy"].float()
        dx = torch.matmul(dy, w)
        if c["act"] != "none":
            dx = dx * _act_slope(c["act"], s["z_below"].float())
        if s["dresidual"] is not None:
            dx = dx + s["dresidual"].float()
        out += [torch.matmul(dy.t(), x), dy.sum(0), dx.to(dt)]
    return out


def _distill(s):
    c = s["case"]
    tau = c["temperature"]
    if own:
        import paper_1712_04432_amd as imbd
        imbd.distill_xent(s["logits"], s["ids"], s["teacher"], s["inv_batch"], s["loss"], s["row_loss"],
                          dlogits=s["dlogits"], temperature=tau, lse=s["lse"], weight=s["weight"], ws=s["ws"])
        return [s["loss"], s["row_loss"]] + ([s["dlogits"]] if c["grad"] else [])
    z = s["logits"].float() * (1.0 / tau)
    peak = z.amax(1, keepdim=True)
    lse = peak + torch.log(torch.exp(z - peak).sum(1, keepdim=True))
    there = s["ids"] >= 0
    at = s["ids"].clamp(min=0).long()
    t = torch.where(there, s["teacher"] * (1.0 / tau), torch.full_like(s["teacher"], -math.inf))
    if s["lse"] is None:
        top = t.amax(1, keepdim=True)
        logp = t - (top + torch.log(torch.exp(t - top).sum(1, keepdim=True)))
    else:
        logp = t - s["lse"][:, None]
    p = torch.exp(logp)
    terms = torch.where(there, p * (logp - (z.gather(1, at) - lse)), torch.zeros_like(p))
    weight = 1.0 if s["weight"] is None else s["weight"]
    row = (tau * tau) * weight * terms.sum(1)
    out = [(row.sum() * s["inv_batch"]).reshape(1), row]
    if c["grad"]:
        dz = torch.exp(z - lse) * p.sum(1, keepdim=True)
        dz.scatter_add_(1, at, -p)
        scale = s["inv_batch"] * tau * weight
        out.append((dz * (scale if s["weight"] is None else scale[:, None])).to(_dtype(c)))
    return out


def _logprobs(s):
    c = s["case"]
    n, tau = c["top"], c["temperature"]
    if own:
        import paper_1712_04432_amd as imbd
        imbd.token_logprobs(s["logits"], s["tokens"], s["logp"], entropy=s["entropy"], lse=s["lse"],
                            top_ids=s["top_ids"], top_logp=s["top_logp"], temperature=tau, ws=s["ws"])
        out = [s["logp"], s["entropy"], s["lse"]] + ([s["top_ids"], s["top_logp"]] if n else [])
        if c["bwd"]:
            imbd.token_logprobs_bwd(s["logits"], s["tokens"], s["lse"], s["dlogits"], dlogp=s["dlogp"],
                                    entropy=s["entropy"], dentropy=s["dentropy"], temperature=tau)
            out.append(s["dlogits"])
        return out
    z = s["logits"].float() * (1.0 / tau)
    peak = z.amax(1, keepdim=True)
    lse = peak + torch.log(torch.exp(z - peak).sum(1, keepdim=True))
    logq = z - lse
    q = torch.exp(logq)
    entropy = -(torch.where(q > 0, q * logq, torch.zeros_like(q))).sum(1, keepdim=True)
    there = (s["tokens"] >= 0)[:, None]
    at = s["tokens"].clamp(min=0).long()[:, None]
    logp = torch.where(there, logq.gather(1, at), torch.zeros_like(lse))
    out = [logp.squeeze(1), entropy.squeeze(1), lse.squeeze(1)]
    if n:
        values, ids = torch.sort(s["logits"], dim=1, descending=True, stable=True)  # ties go to the lowest token
        out += [ids[:, :n].to(torch.int32), values[:, :n].float() * (1.0 / tau) - lse]
    if c["bwd"]:
        dlogp = torch.where(there, s["dlogp"][:, None], torch.zeros_like(lse))
        dz = -q * dlogp - torch.where(q > 0, q * (logq + entropy), torch.zeros_like(q)) * s["dentropy"][:, None]
        dz.scatter_add_(1, at, dlogp)
        out.append((dz * (1.0 / tau)).to(_dtype(c)))
    return out


# ------------------------------------------------------------------------------------ what a pass needs
def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "linear":
        B, d_in, d_out = case["B"], case["d_in"], case["d_out"]
        byte, flop = d_in * d_out * es + B * d_in * es, 0
        if case["pass"] != "bwd":
            byte += B * d_out * es * (1 + case["residual"] + case["keep"]) + d_out * 4 * case["bias"]
            flop += 2 * B * d_in * d_out
        if case["pass"] != "fwd":
            byte += B * d_out * es + d_in * d_out * 4 + d_out * 4
            byte += B * d_in * es * (1 + case["residual"] + (case["act"] != "none"))
            flop += 4 * B * d_in * d_out
        return {"bytes": byte, "flops": flop}
    B, V = case["B"], case["V"]
    if case["kind"] == "distill":
        byte = B * V * es + B * case["K"] * 8 + B * 4 * (1 + case["mass"] + (case["pad"] > 0)) + 4
        return {"bytes": byte + (B * V * es if case["grad"] else 0), "flops": B * V * (8 if case["grad"] else 4)}
    byte, flop = B * V * es + B * 16 + B * case["top"] * 8, 6 * B * V
    if case["bwd"]:
        # (a pass of its own, after what the caller makes of the first one's results: it reads the logits again)
        byte += 2 * B * V * es + B * 20
        flop += 8 * B * V
    return {"bytes": byte, "flops": flop}


# ------------------------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "distill": _exact_distill, "logprobs": _exact_logprobs}[case["kind"]](s, case)


def _exact_linear(s, c):
    f64 = torch.float64
    name = c["act"]

    def f(v):
        if name == "relu":
            return torch.relu(v)
        if name == "gelu":
            return v * torch.special.ndtr(v)
        if name == "gelu_tanh":
            return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
        return v * torch.sigmoid(v) if name == "silu" else v

    def slope(v):
        if name == "relu":
            return torch.heaviside(v, torch.zeros((), dtype=f64, device=DEV))
        if name == "gelu":
            return torch.special.ndtr(v) + v * torch.exp(-v.square() / 2) / math.sqrt(2 * math.pi)
        if name == "gelu_tanh":
            a = 2 * math.sqrt(2 / math.pi)
            p = torch.sigmoid(a * (v + 0.044715 * v ** 3))
            return p + v * p * (1 - p) * a * (1 + 0.134145 * v ** 2)
        p = torch.sigmoid(v)
        return p + v * p * (1 - p)

    w, x = s["w"].to(f64), s["x"].to(f64)
    out = []
    if c["pass"] != "bwd":
        z = x @ w.t()
        if c["bias"]:
            z += s["bias"].to(f64)
        y = f(z)
        if c["residual"]:
            y = y + s["residual"].to(f64)
        out += [y, z] if c["keep"] else [y]
    if c["pass"] != "fwd":
        dy = s["dy"].to(f64)
        dw, db, dx = dy.t() @ x, dy.sum(0), dy @ w
        if name != "none":
            dx *= slope(s["z_below"].to(f64))
        if c["residual"]:
            dx += s["dresidual"].to(f64)
        out += [dw, db, dx]
    return out


def _exact_distill(s, c):
    f64 = torch.float64
    B, V, tau = c["B"], c["V"], c["temperature"]
    row = torch.zeros(B, dtype=f64, device=DEV)
    dz = torch.empty(B, V, dtype=f64, device=DEV) if c["grad"] else None
    per = max(1, 40_000_000 // V)
    for a in range(0, B, per):
        b = min(B, a + per)
        logq = torch.log_softmax(s["logits"][a:b].to(f64) / tau, 1)
        t = (s["teacher"][a:b].to(f64) / tau).masked_fill(s["ids"][a:b] < 0, -math.inf)
        logp = torch.log_softmax(t, 1) if s["lse"] is None else t - s["lse"][a:b].to(f64)[:, None]
        p = logp.exp()
        full = torch.zeros(b - a, V, dtype=f64, device=DEV)
        rows, cols = torch.nonzero(s["ids"][a:b] >= 0, as_tuple=True)
        v = s["ids"][a:b][rows, cols].long()
        full.index_put_((rows, v), p[rows, cols], accumulate=True)
        row[a:b].index_add_(0, rows, p[rows, cols] * (logp[rows, cols] - logq[rows, v]))
        row[a:b] *= tau ** 2
        weight = torch.ones(b - a, dtype=f64, device=DEV) if s["weight"] is None else s["weight"][a:b].to(f64)
        row[a:b] *= weight
        if c["grad"]:
            dz[a:b] = (logq.exp() * full.sum(1, keepdim=True) - full) * (weight * tau * s["inv_batch"])[:, None]
    loss = (row.sum() * s["inv_batch"]).reshape(1)
    return [loss, row, dz] if c["grad"] else [loss, row]


def _exact_logprobs(s, c):
    f64 = torch.float64
    B, V, n, tau = c["B"], c["V"], c["top"], c["temperature"]
    logp, entropy, lse = (torch.zeros(B, dtype=f64, device=DEV) for _ in range(3))
    ids = torch.zeros(B, n, dtype=torch.int64, device=DEV)
    best = torch.zeros(B, n, dtype=f64, device=DEV)
    dz = torch.empty(B, V, dtype=f64, device=DEV) if c["bwd"] else None
    per = max(1, 40_000_000 // V)
    for a in range(0, B, per):
        b = min(B, a + per)
        z = s["logits"][a:b].to(f64)
        lse[a:b] = torch.logsumexp(z / tau, 1)
        logq = torch.log_softmax(z / tau, 1)
        q = logq.exp()
        entropy[a:b] = torch.special.entr(q).sum(1)
        rows = torch.nonzero(s["tokens"][a:b] >= 0).squeeze(1)
        v = s["tokens"][a:b][rows].long()
        logp[a + rows] = logq[rows, v]
        if n:
            order = torch.argsort(z, dim=1, descending=True, stable=True)[:, :n]
            ids[a:b], best[a:b] = order, logq.gather(1, order)
        if c["bwd"]:
            g = torch.zeros(b - a, dtype=f64, device=DEV)
            g[rows] = s["dlogp"][a + rows].to(f64)
            h = s["dentropy"][a:b].to(f64)
            d = -g[:, None] * q + h[:, None] * (torch.special.entr(q) - q * entropy[a:b, None])
            d[rows, v] += g[rows]
            dz[a:b] = d / tau
    out = [logp, entropy, lse] + ([ids, best] if n else [])
    return out + [dz] if c["bwd"] else out
