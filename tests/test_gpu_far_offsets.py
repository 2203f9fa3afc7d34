"""Tensors of more than 2^31 elements and the largest numbers of rows, through a layer's products and what its logits are for.

Layers: whole numbers, bit for bit (as in tests/test_gpu_linear_exact.py), compared in slices. Logits: the last rows against a call
on them alone, which takes the same kernels."""
import pytest

from tests.test_gpu_expert import _dt, _gen
from tests.test_gpu_vocab import _ws

pytestmark = pytest.mark.gpu

SLICE = 1 << 27  # elements at once


@pytest.fixture(autouse=True)
def _released(dev):
    import torch
    yield
    torch.cuda.empty_cache()


def _fill(t, most, g):
    import torch
    n = max(1, SLICE // t.shape[1])
    for r in range(0, t.shape[0], n):
        part = t[r:r + n]
        part.copy_(torch.randint(-most, most + 1, part.shape, generator=g, device=t.device, dtype=torch.int8))
    return t


def _same(got, ref_of, what):
    """ref_of(slice of rows): what they have to be."""
    n = max(1, SLICE // max(got.shape[1], 32))
    for r in range(0, got.shape[0], n):
        rows = slice(r, min(r + n, got.shape[0]))
        bad = got[rows] != ref_of(rows).to(got.dtype)
        assert not bad.any(), (what, r, int(bad.sum()), bad.nonzero()[:4].tolist())


# rows past 2^31 elements: any-size kernel (which takes as many as a launch has tiles), large tiles; weights past 2^31 elements: few rows,
# large tiles, any size
@pytest.mark.parametrize("dtype,B,d_out,d_in", [("bf16", 2 ** 29 + 37, 3, 5), ("bf16", 2 ** 28 + 37, 8, 16), ("f32", 2 ** 27 + 5, 2, 33),
                                                ("bf16", 8, 2 ** 19 + 8, 4104), ("bf16", 300, 2 ** 19 + 8, 4104), ("f32", 40, 2 ** 19 + 3, 4101)])
def test_layers(imbd, dev, dtype, B, d_out, d_in):
    import torch
    g, dt = _gen(B, dev), _dt(dtype)

    def e(*s, t=dt):
        return torch.empty(*s, dtype=t, device=dev)

    w, x, dy = _fill(e(d_out, d_in), 1, g), _fill(e(B, d_in), 2, g), _fill(e(B, d_out), 1, g)
    if B > 2 ** 20:  # (sums over the rows have to stay under 2^24)
        dy[1000:-1000] = 0
    if d_out > 2 ** 18:
        dy[:, 3000:-3000] = 0
    code = imbd.dtype_code(dt)
    ws = [torch.full((max(8, imbd.linear_workspace_bytes(k, code, d_out, d_in, B)),), 255, dtype=torch.uint8, device=dev) for k in (0, 1)]
    y = torch.full((B, d_out), 7.0, dtype=dt, device=dev)
    imbd.linear_fwd(w, x, y, act="relu", ws=ws[0])
    if d_out > B:
        _same(y.t(), lambda r: (w[r].float() @ x.float().t()).clamp(min=0), "y")
    else:
        _same(y, lambda r: (x[r].float() @ w.float().t()).clamp(min=0), "y")
    del y
    dx, dw, db = e(B, d_in), e(d_out, d_in, t=torch.float32), e(d_out, t=torch.float32)
    imbd.linear_bwd(w, dy, x, dw=dw, db=db, dx=dx, ws=ws[1])
    if B > 2 ** 20:
        _same(dx, lambda r: dy[r].float() @ w.float(), "dx")
        ends = [torch.cat([t[:1000], t[-1000:]]).double() for t in (dy, x)]
        assert torch.equal(dw.double(), ends[0].t() @ ends[1]) and torch.equal(db.double(), ends[0].sum(0))
    else:
        ends = [torch.cat([t[:3000], t[-3000:]]).double() for t in (dy.t(), w)]
        assert torch.equal(dx, (ends[0].t() @ ends[1]).to(dt))
        _same(dw, lambda r: dy[:, r].t().float() @ x.float(), "dw")
        assert torch.equal(db.double(), dy.double().sum(0))


def test_activations_of_far_elements(imbd, dev):
    import torch
    B, d = 2 ** 20 + 3, 2051
    g = _gen(1, dev)
    dy, z = (_fill(torch.empty(B, d, dtype=torch.bfloat16, device=dev), 2, g) for _ in range(2))
    dz = torch.full_like(dy, 7.0)
    imbd.act_bwd(dy, z, dz, "relu")
    _same(dz, lambda r: dy[r].float() * (z[r].float() > 0), "dz")


def _logits(B, V, dtype, dev):
    import torch
    z = torch.empty(B, V, dtype=_dt(dtype), device=dev)
    n = max(1, SLICE // V)
    g = _gen(V, dev)
    for r in range(0, B, n):
        z[r:r + n] = torch.randn(z[r:r + n].shape, generator=g, device=dev) * 3
    return z


@pytest.mark.parametrize("dtype,out,B,V", [("bf16", "bf16", 70001, 65537), ("f32", "f32", 40001, 65536), ("f32", "bf16", 70003, 32771),
                                           ("bf16", "bf16", 2 ** 24 - 1, 8), ("f32", "bf16", 2 ** 24 - 1, 5), ("bf16", "bf16", 2 ** 22, 264)])
def test_logits(imbd, dev, dtype, out, B, V):
    import torch
    z = _logits(B, V, dtype, dev)
    g = _gen(1, dev)
    # (a row's sums are added in the order of its 16-byte chunks, so the rows apart begin at the same place in 16 bytes)
    K, n, last = 2, 3, 1000 + (B - 1000) % 8
    ids = torch.randint(0, V, (B, K), generator=g, device=dev, dtype=torch.int32)
    t = torch.randn(B, K, generator=g, device=dev)
    tokens = torch.randint(0, V, (B,), generator=g, device=dev, dtype=torch.int32)
    up = torch.randn(B, generator=g, device=dev)

    def run(z, ids, t, tokens, up, in_place):
        B = z.shape[0]
        f = lambda *s: torch.full(s, 7.0, device=dev)  # noqa: E731
        o = dict(logp=f(B), ent=f(B), lse=f(B), top=f(B, n), ids=torch.full((B, n), 7, dtype=torch.int32, device=dev), loss=f(1), row=f(B))
        imbd.token_logprobs(z, tokens, o["logp"], entropy=o["ent"], lse=o["lse"], top_ids=o["ids"], top_logp=o["top"],
                            ws=_ws(imbd.token_logprobs_workspace_bytes(B, V, n), dev))
        o["dl"] = torch.full(z.shape, 7.0, dtype=_dt(out), device=dev)
        imbd.token_logprobs_bwd(z, tokens, o["lse"], o["dl"], dlogp=up, entropy=o["ent"], dentropy=up)
        o["dz"] = z if in_place else torch.full(z.shape, 7.0, dtype=_dt(out), device=dev)
        imbd.distill_xent(z, ids, t, 1.0 / B, o["loss"], o["row"], dlogits=o["dz"], ws=_ws(imbd.distill_workspace_bytes(B, V, K), dev))
        torch.cuda.synchronize()
        return o

    tail = [v[-last:].clone() for v in (z, ids, t, tokens, up)]
    whole = run(z, ids, t, tokens, up, dtype == out)
    part = run(*tail, False)
    for k, v in part.items():
        if k == "loss":
            continue
        got = whole[k][-last:]
        if k == "dz":  # (its scale is 1 / B: powers of two of it only would be the same bits)
            err = (got.double() * B - v.double() * last).abs()
            assert (err <= 2 ** -6 * (v.double() * last).abs() + 2.0 ** -100 * B).all(), k
        else:
            assert torch.equal(got, v), k
    total = whole["row"].double().mean().item()
    assert abs(whole["loss"].item() - total) <= 1e-6 * whole["row"].double().abs().mean().item() * max(1, B / 2 ** 18)
