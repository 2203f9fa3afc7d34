"""distill_xent, token_logprobs and its gradient against their formulas in 64 bits.

Tolerances are bounds by arithmetic, not fits. With h = 2^-24 (half a step of fp32), d a logit's distance from the row's
reference in natural units, |d| at most D + 12 off the reference that a kernel may use (up to 16 octaves under the
largest logit):
* the scaled distance is off by 5 h |d| (its difference, the factor log2(e) / temperature and two products), a term
  e^d by that and 2 h of its own, and a sum of V terms of one sign by the length of its longest chain, at most V / 256 + 40
  additions;
* so ln s is off by rho = h (5 mean|d| + V / 256 + 48), mean over q, and 2 h |ln s| for the logarithm;
* what is stored as bf16 is off by half a step more, 2^-8 of the value."""
import numpy as np
import pytest

from tests.test_gpu_expert import _dt, _gen, _padded

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TINY = 2.0 ** -120  # results under the smallest normal number may be 0


def _logits(dev, B, V, dtype, kind="normal", pad=0, seed=0):
    """[B][V] in surroundings of NaN (pad: elements between the rows)."""
    import torch
    g = _gen(seed, dev)
    z, whole = _padded((B, V), V + pad, _dt(dtype), dev)
    x = torch.randn(B, V, generator=g, device=dev) * 3
    if kind == "masked":
        x[torch.rand(B, V, generator=g, device=dev) < 0.6] = -float("inf")
        x[:, V // 2] = 1.0  # (something is left)
    elif kind == "one_left":
        x[:] = -float("inf")
        x[torch.arange(B), torch.randint(0, V, (B,), generator=g, device=dev)] = -5.0
    elif kind == "lowest":  # masked by the type's lowest value
        x[torch.rand(B, V, generator=g, device=dev) < 0.6] = torch.finfo(_dt(dtype)).min
        x[:, V - 1] = 2.0
    elif kind == "all_lowest":
        x[:] = torch.finfo(_dt(dtype)).min
    elif kind == "ties":
        x = torch.randint(-2, 3, (B, V), generator=g, device=dev).float()
    elif kind == "constant":
        x[:] = 4.25
    elif kind == "ascending":
        x = (torch.arange(V, device=dev).float() / V * 20 - 10).expand(B, V)
    elif kind == "descending":
        x = (torch.arange(V, device=dev).float() / V * -20 + 10).expand(B, V)
    elif kind == "peaked":
        x[:, V // 3] = 60.0
    elif kind == "large":
        x *= 1e4
    else:
        assert kind == "normal"
    z.copy_(x)
    return z


class Exact:
    """A row's statistics in 64 bits."""

    def __init__(self, z, temperature):
        import torch
        self.t = temperature
        self.z = z.double() / temperature
        top = self.z.amax(1, keepdim=True)
        self.top = top.squeeze(1)
        self.ln_s = torch.logsumexp(self.z - top, 1)  # (by differences: logits of 1e38 leave lse itself no digits)
        self.lse = self.top + self.ln_s
        self.logq = (self.z - top) - self.ln_s[:, None]
        self.q = self.logq.exp()
        self.H = torch.where(self.q > 0, -self.q * self.logq, torch.zeros_like(self.q)).sum(1)
        V = z.shape[1]
        d = (top - self.z).clamp(max=1e30) + 12
        mean = torch.where(self.q > 0, self.q * d, torch.zeros_like(d)).sum(1)
        square = torch.where(self.q > 0, self.q * d * d, torch.zeros_like(d)).sum(1)
        self.d = torch.where(self.z > -float("inf"), d, torch.zeros_like(d))
        ln_s = self.ln_s.abs() + 12
        self.rho = H * (5 * mean + V / 256 + 48)
        self.tol_ln = self.rho + 2 * H * ln_s
        self.tol_lse = self.tol_ln + 4 * H * (self.top.abs() + 12 + self.lse.abs())
        self.tol_H = 2 * self.rho * (1 + mean) + 5 * H * square + 8 * H * (ln_s + mean + self.H)

    def tol_logq(self, z):
        """Of log q of logits z / t [B] or [B][n]."""
        top, tol = (v if z.dim() == 1 else v[:, None] for v in (self.top, self.tol_ln))
        return tol + 5 * H * ((top - z).abs() + 12) + 2 * H * self.log_q(z).abs()

    def log_q(self, z):
        """log q of logits z / t [B] or [B][n]."""
        top, ln_s = (v if z.dim() == 1 else v[:, None] for v in (self.top, self.ln_s))
        return (z - top) - ln_s


def _near(got, ref, tol, what):
    import torch
    got, ref = got.double(), ref.double()
    same = (got == ref) | (got.isnan() & ref.isnan())
    same |= (got.abs() == float("inf")) & (got.sign() == ref.sign()) & (ref.abs() + tol >= torch.finfo(torch.float32).max)
    bad = ~(same | ((got - ref).abs() <= tol))
    assert not bad.any(), (what, int(bad.sum()), bad.numel(), ((got - ref).abs() / tol)[bad].max().item(),
                           got[bad][:4].tolist(), ref[bad][:4].tolist())


def _ws(nbytes, dev, fill=255):
    import torch
    return torch.full((nbytes,), fill, dtype=torch.uint8, device=dev) if nbytes else None


def _tokens(dev, B, V, seed=1):
    import torch
    t = torch.randint(0, V, (B,), generator=_gen(seed, dev), device=dev, dtype=torch.int32)
    t[::5] = -1
    t[0] = V - 1
    return t


def _run_logprobs(imbd, z, tokens, n, temperature=1.0):
    import torch
    B, V = z.shape
    dev = z.device
    logp, ent, lse = (torch.full((B,), 7.0, device=dev) for _ in range(3))
    ids = torch.full((B, n), 77, dtype=torch.int32, device=dev) if n else None
    top = torch.full((B, n), 7.0, device=dev) if n else None
    ws = _ws(imbd.token_logprobs_workspace_bytes(B, V, n), dev)
    imbd.token_logprobs(z, tokens, logp, entropy=ent, lse=lse, top_ids=ids, top_logp=top, temperature=temperature, ws=ws)
    return logp, ent, lse, ids, top


def _check_logprobs(imbd, z, tokens, n, temperature=1.0):
    import torch
    B, V = z.shape
    logp, ent, lse, ids, top = _run_logprobs(imbd, z, tokens, n, temperature)
    torch.cuda.synchronize()
    x = Exact(z, temperature)
    at = tokens.clamp(0, V - 1).long()[:, None]
    zt = x.z.gather(1, at).squeeze(1)
    ref = torch.where(tokens < 0, torch.zeros_like(zt), x.log_q(zt))
    _near(logp, ref, x.tol_logq(zt), "logp")
    _near(lse, x.lse, x.tol_lse, "lse")
    _near(ent, x.H, x.tol_H, "entropy")
    if n:
        order = torch.argsort(z.float(), dim=1, descending=True, stable=True)[:, :n]
        if n > V:
            order = torch.nn.functional.pad(order, (0, n - V))
        zs = x.z.gather(1, order)
        there = (zs > -float("inf")) & (torch.arange(n, device=z.device) < V)
        assert torch.equal(ids, torch.where(there, order, torch.full_like(order, -1)).to(torch.int32))
        ref = torch.where(there, x.log_q(zs), torch.full_like(zs, -float("inf")))
        _near(top, ref, x.tol_logq(zs), "top_logp")


SIZES = [(1, 1), (3, 2), (5, 7), (2, 8), (4, 63), (3, 64), (2, 255), (2, 257), (300, 1000), (7, 1023), (3, 4099),
         (2, 32768), (3, 50021), (1, 131072), (2, 262147)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,V", SIZES)
def test_logprobs_sizes(imbd, dev, B, V, dtype):
    z = _logits(dev, B, V, dtype, pad=(B * 3 + V) % 5, seed=V)
    for n in (0, 1, 5, 64):
        _check_logprobs(imbd, z, _tokens(dev, B, V), n, 0.7 if n == 5 else 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["masked", "one_left", "lowest", "all_lowest", "ties", "constant", "ascending", "descending",
                                  "peaked", "large"])
@pytest.mark.parametrize("B,V", [(2, 50), (3, 1000), (2, 9001), (2, 70001), (600, 2100)])
def test_logprobs_values(imbd, dev, B, V, kind, dtype):
    _check_logprobs(imbd, _logits(dev, B, V, dtype, kind, pad=3), _tokens(dev, B, V), 20, 1.0)


def test_logprobs_candidates_in_one_lane(imbd, dev):
    """Rows whose largest logits lie at one stride (any power of two up to 2^14), where one thread may see them all."""
    import torch
    V = 131072
    for stride in [1 << i for i in range(15)] + [2048 * 3, 1000]:
        z = torch.randn(2, V, device=dev, generator=_gen(stride, dev)).to(torch.bfloat16)
        at = (torch.arange(4000, device=dev) * stride + 5) % V
        z[0, at] = 20.0
        z[1, at] = (20.0 + torch.arange(4000, device=dev) % 97).to(torch.bfloat16)
        _check_logprobs(imbd, z, _tokens(dev, 2, V), 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_begin_inside_a_chunk(imbd, dev, dtype):
    """Every place in 16 bytes where a row may begin and end, short rows and rows in parts; the gradient's rows elsewhere."""
    import torch
    for V in (1, 2, 3, 7, 9, 15, 17, 40, 2049, 9001, 20003):
        whole = torch.full((3 * V + 40,), float("nan"), dtype=_dt(dtype), device=dev)
        for start in range(9):
            z = whole[start:start + 3 * V].view(3, V)
            z.copy_(torch.randn(3, V, generator=_gen(start, dev), device=dev) * 3)
            tokens = _tokens(dev, 3, V)
            _check_logprobs(imbd, z, tokens, 5)
            ids, t = _teacher(dev, 3, V, min(V, 4))
            _check_distill(imbd, z, ids, t, dtype)
            g = torch.randn(3, generator=_gen(1, dev), device=dev)
            _, ent, lse, _, _ = _run_logprobs(imbd, z, tokens, 0)
            a = torch.full((3 * V + 9,), 7.0, dtype=_dt(dtype), device=dev)
            b = torch.full((3, V), 7.0, dtype=_dt(dtype), device=dev)
            imbd.token_logprobs_bwd(z, tokens, lse, a[8 - start:8 - start + 3 * V].view(3, V), dlogp=g, entropy=ent, dentropy=g)
            imbd.token_logprobs_bwd(z.clone(), tokens, lse, b, dlogp=g, entropy=ent, dentropy=g)
            assert torch.equal(a[8 - start:8 - start + 3 * V].view(3, V), b), (V, start)
            assert (a[:8 - start] == 7.0).all() and (a[8 - start + 3 * V:] == 7.0).all()
            whole.fill_(float("nan"))


def test_logprobs_many_rows(imbd, dev):
    for dtype in ("bf16", "f32"):
        _check_logprobs(imbd, _logits(dev, 5000, 1037, dtype, "masked"), _tokens(dev, 5000, 1037), 3)
        _check_logprobs(imbd, _logits(dev, 1030, 8192, dtype, pad=8), _tokens(dev, 1030, 8192), 0)


@pytest.mark.parametrize("V", [5, 3001, 100000])
def test_logprobs_not_a_number(imbd, dev, V):
    """NaN, +inf and rows of -inf only make their own row NaN and nobody else's; a token past the end is NaN."""
    import torch
    z = _logits(dev, 6, V, "f32")
    z[1, V // 2] = float("nan")
    z[2, V - 1] = float("inf")
    z[3] = -float("inf")
    tokens = torch.tensor([0, 1, 2, 3, V, 2 ** 31 - 1], dtype=torch.int32, device=dev)
    logp, ent, lse, ids, top = _run_logprobs(imbd, z, tokens, 4)
    torch.cuda.synchronize()
    assert logp.isnan().tolist() == [False, True, True, True, True, True]
    assert ent.isnan().tolist() == [False, True, True, True, False, False]
    assert lse.isnan().tolist() == [False, True, True, False, False, False] and lse[3] == -float("inf")
    assert ids[3].tolist() == [-1] * 4 and (top[3] == -float("inf")).all()
    assert (ids >= -1).all() and (ids < V).all() and ids[2, 0] == V - 1
    ok = z.clone()
    ok[1, V // 2] = -float("inf")
    assert torch.equal(ids[1], _run_logprobs(imbd, ok, tokens, 4)[3][1])  # (a NaN is no alternative)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("B,V", [(1, 1), (3, 7), (5, 64), (4, 1000), (2, 4099), (3, 50021), (2, 131072), (700, 515)])
def test_logprobs_bwd(imbd, dev, B, V, dtype, out):
    import torch
    t = 0.7 if V == 1000 else 1.0
    z = _logits(dev, B, V, dtype, "masked" if V % 2 else "normal", pad=V % 3)
    tokens = _tokens(dev, B, V)
    g, h = (torch.randn(B, generator=_gen(s, dev), device=dev) for s in (3, 4))
    _, ent, lse, _, _ = _run_logprobs(imbd, z, tokens, 0, t)
    x = Exact(z, t)
    logq = torch.where(x.q > 0, x.logq, torch.zeros_like(x.q))
    for use_g, use_h in ((True, True), (True, False), (False, True)):
        dz, whole = _padded((B, V), V + 5, _dt(out), dev, 7.0)
        imbd.token_logprobs_bwd(z, tokens, lse, dz, dlogp=g if use_g else None, entropy=ent if use_h else None,
                                dentropy=h if use_h else None, temperature=t)
        torch.cuda.synchronize()
        gg = (torch.where(tokens >= 0, g, torch.zeros_like(g)) if use_g else torch.zeros_like(g)).double()[:, None]
        hh = (h if use_h else torch.zeros_like(h)).double()[:, None]
        hot = torch.zeros_like(x.q).scatter_(1, tokens.clamp(min=0).long()[:, None], 1.0)
        ref = (gg * (hot - x.q) - hh * x.q * (logq + x.H[:, None])) / t
        # log q is off by dl (as the forward pass's lse, and 4 h for its own scaling of z), q by that and the factor log2(e)
        dl = x.tol_lse[:, None] + 4 * H * (x.z.abs().clamp(max=1e30) * (x.q > 0) + logq.abs())
        dq = x.q * (dl + 4 * H * (1 + logq.abs()))
        inner = logq.abs() + x.H[:, None]
        tol = (gg.abs() * (dq + 4 * H * (hot + x.q)) + hh.abs() * (dq * inner + x.q * (dl + x.tol_H[:, None] + 6 * H * inner))) / t
        tol = tol + 2 * H * ref.abs() + STEP[out] * (ref.abs() + tol) + TINY
        _near(dz, ref, tol, "dlogits")
        assert (whole[:, V:] == 7.0).all()


def test_logprobs_bwd_special_rows(imbd, dev):
    """Zeros where nothing flows back, NaN for a token past the end, and in place of the logits."""
    import torch
    B, V = 6, 3001
    z = _logits(dev, B, V, "bf16", "masked")
    z[3, 5] = float("nan")
    tokens = torch.tensor([5, -1, V, 7, V, 9], dtype=torch.int32, device=dev)
    g = torch.tensor([1.0, 1.0, 1.0, 0.0, 0.0, -2.0], device=dev)
    _, ent, lse, _, _ = _run_logprobs(imbd, z, tokens, 0)
    dz = torch.full_like(z, 7.0)
    imbd.token_logprobs_bwd(z, tokens, lse, dz, dlogp=g)
    assert dz.isnan().all(1).tolist() == [False, False, True, False, False, False]
    assert (dz[[1, 3, 4]] == 0).all() and (dz[[0, 5]] != 0).any(1).all()
    out = z[0] == -float("inf")
    out[5] = False  # (the token's own slope is g (1 - q))
    assert (dz[0, out] == 0).all()
    imbd.token_logprobs_bwd(z, tokens, lse, z, dlogp=g)
    torch.cuda.synchronize()
    assert torch.equal(z.view(torch.int16), dz.view(torch.int16))


def test_logprobs_bwd_against_differences(imbd, dev):
    import torch
    B, V, t, step = 4, 11, 0.7, 2.0 ** -7
    z = _logits(dev, B, V, "f32")
    tokens = _tokens(dev, B, V)
    g, h = (torch.randn(B, generator=_gen(s, dev), device=dev) for s in (3, 4))
    _, ent, lse, _, _ = _run_logprobs(imbd, z, tokens, 0, t)
    dz = torch.empty_like(z)
    imbd.token_logprobs_bwd(z, tokens, lse, dz, dlogp=g, entropy=ent, dentropy=h, temperature=t)

    def f(x):
        logp, ent, _, _, _ = _run_logprobs(imbd, x, tokens, 0, t)
        return (g * logp + h * ent).double()

    for v in range(V):
        up, down = z.clone(), z.clone()
        up[:, v] += step
        down[:, v] -= step
        slope = (f(up) - f(down)) / (up[:, v] - down[:, v]).double()
        # third derivatives of log q and H by z are under 40 / t^3 here (|log q| < 35), and f is off by some 2^-19
        assert ((slope - dz[:, v].double()).abs() <= (g.abs() + h.abs()).double() * (40 / t ** 3 * step ** 2 / 6 + 2.0 ** -19 / step)).all()


# ------------------------------------------------------------------------------------ distillation
def _teacher(dev, B, V, K, seed=2, distinct=True):
    import torch
    g = _gen(seed, dev)
    first = torch.randint(0, V, (B, 1), generator=g, device=dev)
    step = next(p for p in (7919, 101, 3, 1) if V % p or p == 1)
    ids = (first + step * torch.arange(K, device=dev)) % V if distinct else torch.randint(0, V, (B, K), generator=g, device=dev)
    t = torch.randn(B, K, generator=g, device=dev) * 2
    return ids.to(torch.int32), t


def _run_distill(imbd, z, ids, t, out=None, lse=None, weight=None, temperature=1.0, inv_batch=0.25, dz=None):
    import torch
    B, V = z.shape
    dev = z.device
    loss, row = torch.full((1,), 7.0, device=dev), torch.full((B,), 7.0, device=dev)
    whole = None
    if dz is None and out:
        dz, whole = _padded((B, V), V + 3, _dt(out), dev, 7.0)
    ws = _ws(imbd.distill_workspace_bytes(B, V, ids.shape[1]), dev)
    imbd.distill_xent(z, ids, t, inv_batch, loss, row, dlogits=dz, temperature=temperature, lse=lse, weight=weight, ws=ws)
    torch.cuda.synchronize()
    assert whole is None or (whole[:, V:] == 7.0).all()
    return loss, row, dz


def _check_distill(imbd, z, ids, t, out="f32", lse=None, weight=None, temperature=1.0, inv_batch=0.25):
    import torch
    B, V = z.shape
    loss, row, dz = _run_distill(imbd, z, ids, t, out, lse, weight, temperature, inv_batch)
    x = Exact(z, temperature)
    there = (ids >= 0) & (t > -float("inf"))
    none = ~there.any(1)
    ts = torch.where(there, t.double() / temperature, torch.full_like(t.double(), -float("inf")))
    lt = torch.logsumexp(ts, 1) if lse is None else lse.double()
    logp = torch.where(there, ts - lt[:, None], torch.full_like(ts, -float("inf")))
    p = torch.where(there, logp.exp(), torch.zeros_like(ts))
    logp = torch.where(there, logp, torch.zeros_like(ts))
    at = ids.clamp(min=0).long()
    logq = x.logq.gather(1, at)
    w = torch.ones(B, device=z.device).double() if weight is None else weight.double()
    each = torch.where(p > 0, p * (logp - logq), torch.zeros_like(p))
    off = none | (w == 0)
    ref = torch.where(off, torch.zeros_like(w), w * temperature ** 2 * each.sum(1))
    # log p is off by 3 h of the scaled logit, the logsumexp's rho (K + 40 additions, and the terms') and 2 h of itself
    ta = ts.abs().masked_fill(~there, 0)
    dlp = 3 * H * ta + H * (5 * ta.amax(1, keepdim=True) * 2 + 300) + 2 * H * (logp.abs() + lt.abs()[:, None])
    dlq = x.tol_logq(x.z.gather(1, at))
    K = ids.shape[1]
    dp = p * (dlp + 2 * H)
    size = (p * (logp.abs() + logq.abs())).nan_to_num(0, 0, 0)
    tol = w.abs() * temperature ** 2 * (dp * (logp - logq).abs().nan_to_num(0, 0, 0) + p * (dlp + dlq.nan_to_num(0, 0, 0)) +
                                        (K / 4 + 24) * H * size).sum(1) + TINY
    _near(row, ref, tol, "row_loss")
    total = (row.double().sum() * inv_batch).reshape(1)
    if row.double().sum() > torch.finfo(torch.float32).max:  # (the sum is fp32's: losses at masked tokens of 1e38)
        total = total + float("inf")
    _near(loss, total, inv_batch * (B / 256 + 12) * H * row.double().abs().sum() + TINY, "loss")
    if out:
        full = torch.zeros_like(x.q).scatter_add_(1, at, p)
        dfull = torch.zeros_like(x.q).scatter_add_(1, at, dp + (K + 4) * H * p)
        S, dS = p.sum(1, keepdim=True), (dp + 40 * H * p).sum(1, keepdim=True)
        scale = (inv_batch * w * temperature)[:, None]
        g = torch.where(off[:, None], torch.zeros_like(x.q), scale * (x.q * S - full))
        dq = x.q * (x.rho[:, None] + 5 * H * x.d + 6 * H)
        tol = scale.abs() * (dq * S + x.q * dS + dfull + 4 * H * (x.q * S + full)) * (1 + 4 * H) + TINY
        _near(dz, g, tol + 4 * H * g.abs() + STEP[out] * (g.abs() + tol), "dlogits")
    return loss, row, dz


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("B,V,K", [(1, 1, 1), (3, 2, 2), (2, 9, 5), (5, 64, 64), (300, 1000, 8), (3, 4099, 256), (2, 32768, 50),
                                   (2, 50021, 20), (1, 131072, 64), (2, 150001, 7), (2, 262147, 128), (530, 8200, 3)])
def test_distill_sizes(imbd, dev, B, V, K, dtype, out):
    import torch
    z = _logits(dev, B, V, dtype, pad=V % 4, seed=K)
    ids, t = _teacher(dev, B, V, K)
    _check_distill(imbd, z, ids, t, out)
    _check_distill(imbd, z, ids, t, None, temperature=2.0)
    lse = torch.logsumexp(t / 0.7, 1) + 0.3
    weight = torch.rand(B, generator=_gen(5, dev), device=dev)
    weight[B // 2] = 0.0
    _check_distill(imbd, z, ids, t, out, lse=lse, weight=weight, temperature=0.7, inv_batch=1.0 / B)


@pytest.mark.parametrize("dtype,V", [("bf16", 70003), ("bf16", 98301), ("bf16", 150001), ("bf16", 180224), ("bf16", 180233),
                                     ("f32", 33001), ("f32", 75003), ("f32", 90112), ("f32", 90117)])
def test_distill_long_rows_in_registers(imbd, dev, dtype, V):
    """Enough rows that the long ones stay in registers, up to the longest that fit and just past it."""
    z = _logits(dev, 97, V, dtype, pad=V % 4, seed=V % 1000)
    ids, t = _teacher(dev, 97, V, 9)
    _check_distill(imbd, z, ids, t, dtype, temperature=0.9)


@pytest.mark.parametrize("kind", ["masked", "lowest", "one_left", "all_lowest", "ties", "peaked", "large"])
@pytest.mark.parametrize("B,V", [(3, 60), (2, 9001), (2, 140000), (600, 2100)])
def test_distill_values(imbd, dev, B, V, kind):
    """Entries on masked tokens make the loss infinite; entries that are missing or -inf, and the same id twice."""
    import torch
    z = _logits(dev, B, V, "f32", kind)
    ids, t = _teacher(dev, B, V, 9, distinct=False)
    ids[0, :3] = ids[0, 3]
    ids[1, 4:] = -1
    t[1, 5] = float("nan")  # (of no entry: not read)
    t[0, 8] = -float("inf")
    _check_distill(imbd, z, ids, t)


@pytest.mark.parametrize("V", [40, 5000, 140000])
def test_distill_special_rows(imbd, dev, V):
    """Rows without entries or weight are zeros whatever they hold, ids past the end and values that are no numbers make
    their own row NaN (and the loss)."""
    import torch
    B = 9
    z = _logits(dev, B, V, "bf16")
    ids, t = _teacher(dev, B, V, 4)
    weight = torch.ones(B, device=dev)
    ids[0] = -1
    z[0, 3] = float("nan")
    t[1] = -float("inf")
    weight[2] = 0
    z[2] = float("nan")
    ids[2, 0] = V
    ids[3, 1] = V
    z[4, V - 1] = float("nan")
    z[5, 0] = float("inf")
    z[6] = -float("inf")
    t[7, 2] = float("nan")
    want = [False, False, False, True, True, True, True, True, False]
    loss, row, dz = _run_distill(imbd, z, ids, t, "bf16", weight=weight)
    assert row.isnan().tolist() == want and dz.isnan().all(1).tolist() == want and dz.isnan().any(1).tolist() == want
    assert loss.isnan().all() and (row[:3] == 0).all() and (dz[:3] == 0).all()
    weight[3:8] = 0
    loss, row, dz = _run_distill(imbd, z, ids, t, "bf16", weight=weight)
    assert row[8] > 0 and torch.equal(row[:8], torch.zeros(8, device=dev)) and (dz[:8] == 0).all()
    assert (loss == 0.25 * row[8]).all()


def test_distill_of_no_rows(imbd, dev):
    import torch
    loss, row, _ = _run_distill(imbd, torch.empty(0, 10, device=dev), torch.empty(0, 2, dtype=torch.int32, device=dev),
                                torch.empty(0, 2, device=dev))
    assert loss.item() == 0.0
    assert _run_logprobs(imbd, torch.empty(0, 10, device=dev), torch.empty(0, dtype=torch.int32, device=dev), 3)[0].numel() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,V", [(3, 1000), (2, 90000), (600, 3000), (2, 200000)])
def test_distill_in_place(imbd, dev, B, V, dtype):
    import torch
    z = _logits(dev, B, V, dtype, pad=6)
    ids, t = _teacher(dev, B, V, 30, distinct=False)
    a = _run_distill(imbd, z, ids, t, dtype)
    b = _run_distill(imbd, z, ids, t, dz=z)
    assert torch.equal(a[2], b[2]) and torch.equal(a[1], b[1]) and torch.equal(a[0], b[0])


def test_distill_with_the_label_alone_is_softmax_xent(imbd, dev):
    """One entry: p = 1, the loss is the cross entropy of its token."""
    import torch
    B, V = 64, 1000
    z = _logits(dev, B, V, "f32")
    labels = torch.randint(0, V, (B,), generator=_gen(9, dev), device=dev, dtype=torch.int32)
    loss, row, dz = _run_distill(imbd, z, labels[:, None].contiguous(), torch.randn(B, 1, device=dev), "f32", inv_batch=1 / B)
    l2, r2, d2 = torch.zeros(1, device=dev), torch.zeros(B, device=dev), torch.zeros(B, V, device=dev)
    imbd.softmax_xent(z, labels, 1 / B, l2, r2, d2)
    assert torch.allclose(row, r2, rtol=0, atol=64 * H * r2.abs().max().item())
    assert torch.allclose(dz, d2, rtol=0, atol=64 * H / B) and abs(loss.item() - l2.item()) <= 64 * H * l2.item()


def test_distill_against_differences(imbd, dev):
    import torch
    B, V, K, t, step = 3, 9, 4, 1.5, 2.0 ** -6
    z = _logits(dev, B, V, "f32")
    ids, teacher = _teacher(dev, B, V, K, distinct=False)
    _, row0, dz = _run_distill(imbd, z, ids, teacher, "f32", temperature=t, inv_batch=1.0)
    for v in range(V):
        up, down = z.clone(), z.clone()
        up[:, v] += step
        down[:, v] -= step
        f = [_run_distill(imbd, x, ids, teacher, temperature=t, inv_batch=1.0)[1].double() for x in (up, down)]
        slope = (f[0] - f[1]) / (up[:, v] - down[:, v]).double()
        # the loss's third derivative is under t^2 / t^3, and its values off by some 2^-18
        assert ((slope - dz[:, v].double()).abs() <= step ** 2 / 6 / t + 2.0 ** -18 / step).all()


# ------------------------------------------------------------------------------------ how they are called
@pytest.mark.parametrize("B,V", [(4, 140000), (700, 3001)])
def test_results_repeat_on_another_stream_and_in_a_graph(imbd, dev, B, V):
    """The same bits on every run, on a stream of the caller's and replayed from a graph after the inputs changed."""
    import torch
    z = _logits(dev, B, V, "bf16")
    ids, t = _teacher(dev, B, V, 16)
    tokens = _tokens(dev, B, V)
    g = torch.randn(B, generator=_gen(3, dev), device=dev)
    n = 10
    o = dict(loss=torch.zeros(1, device=dev), row=torch.zeros(B, device=dev), dz=torch.zeros_like(z), logp=torch.zeros(B, device=dev),
             ent=torch.zeros(B, device=dev), lse=torch.zeros(B, device=dev), ids=torch.zeros(B, n, dtype=torch.int32, device=dev),
             top=torch.zeros(B, n, device=dev), dl=torch.zeros_like(z))
    ws = _ws(max(imbd.distill_workspace_bytes(B, V, 16), imbd.token_logprobs_workspace_bytes(B, V, n), 8), dev)

    def call():
        imbd.distill_xent(z, ids, t, 0.5, o["loss"], o["row"], dlogits=o["dz"], ws=ws)
        imbd.token_logprobs(z, tokens, o["logp"], entropy=o["ent"], lse=o["lse"], top_ids=o["ids"], top_logp=o["top"], ws=ws)
        imbd.token_logprobs_bwd(z, tokens, o["lse"], o["dl"], dlogp=g, entropy=o["ent"], dentropy=g)

    def take():
        torch.cuda.synchronize()
        out = {k: v.clone() for k, v in o.items()}
        for v in o.values():
            v.fill_(7)
        torch.cuda.synchronize()
        return out

    call()
    first = take()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    other = take()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        graph.replay()
        again = take()
        for k in first:
            assert torch.equal(first[k], again[k]) and torch.equal(first[k], other[k]), k
    z.copy_(_logits(dev, B, V, "bf16", seed=9))
    call()
    eager = take()
    for _ in range(2):
        graph.replay()
        again = take()
        for k in first:
            assert torch.equal(eager[k], again[k]), k


def test_tensors_elsewhere_are_refused(imbd, dev):
    import torch
    z, tok = torch.zeros(2, 8, device=dev), torch.zeros(2, dtype=torch.int32, device=dev)
    out = torch.zeros(2, device=dev)
    for call in (lambda: imbd.token_logprobs(z.cpu(), tok, out), lambda: imbd.token_logprobs(z, tok.cpu(), out),
                 lambda: imbd.token_logprobs(z, tok, out, ws=torch.zeros(8)),
                 lambda: imbd.token_logprobs(z.t(), tok, out), lambda: imbd.token_logprobs(z[:, ::2], tok, out),
                 lambda: imbd.token_logprobs_bwd(z, tok, out, z.cpu()),
                 lambda: imbd.distill_xent(z, tok[:, None].cpu(), z[:, :1].contiguous(), 1.0, out[:1], out)):
        with pytest.raises((ValueError, TypeError)):
            call()
    with pytest.raises(imbd.ImbdError):
        imbd.token_logprobs(z[:1].expand(2, 8), tok, out)
