"""linear_fwd, linear_bwd and act_bwd against their formulas in 64 bits.

Tolerances are bounds by arithmetic, with h = 2^-24 (half a step of fp32). A product's sum of K terms is off by at most
(K + 2) 2h sum |terms|, whatever the order of its additions. An activation passes that on with a slope of at most 1.13 and
adds its own: exponentials of arguments that are off by some h of their size, a reciprocal and a few products,
* gelu          h (16 + 1.5 z^2 [z < 0]) |y|: the tail is e^(-z^2/2) times a function good to 3 h
* gelu_tanh     h (10 + 6 |v|) |y|, v the exponent;     silu    h (10 + 3 |z|) |y|
* derivatives   32 h (gelu, silu), 64 h (gelu_tanh), absolutely: z^2 phi(z), v p (1 - p) and their like stay under 4.
Storing as bf16 adds half a step, 2^-8 of the value."""
import math

import pytest

from tests.test_gpu_expert import STEP, _dt, _gen, _padded, _randn

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
TINY = 2.0 ** -120
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def _value(act, z):
    import torch
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z * torch.sigmoid(z) if act == "silu" else z


def _slope(act, z):
    import torch
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a = 2 * math.sqrt(2 / math.pi)
        p = torch.sigmoid(a * (z + 0.044715 * z ** 3))
        return p + torch.where(p * (1 - p) > 0, z * p * (1 - p) * a * (1 + 3 * 0.044715 * z * z), torch.zeros_like(z))
    if act == "silu":
        p = torch.sigmoid(z)
        return p + z * p * (1 - p)
    return torch.ones_like(z)


def _value_err(act, z):
    y = _value(act, z).abs()
    if act == "gelu":
        return H * y * (16 + 1.5 * z * z * (z < 0))
    if act == "gelu_tanh":
        return H * y * (10 + 6 * (1.6 * (z + 0.044715 * z ** 3)).abs())
    return H * y * (10 + 3 * z.abs()) if act == "silu" else 0 * y


SLOPE_ERR = {"none": 0.0, "relu": 0.0, "gelu": 32 * H, "gelu_tanh": 64 * H, "silu": 32 * H}


def _near(got, ref, tol, what):
    got = got.double()
    ok = (got == ref) | ((got - ref).abs() <= tol) | (got.isnan() & ref.isnan())
    assert ok.all(), (what, int((~ok).sum()), ok.numel(), ((got - ref).abs() / tol)[~ok].max().item(), got[~ok][:4].tolist(),
                      ref[~ok][:4].tolist())


def _ws(imbd, which, dtype, d_out, d_in, B, dev):
    import torch
    n = imbd.linear_workspace_bytes(which, imbd.dtype_code(_dt(dtype)), d_out, d_in, B)
    return torch.full((n,), 255, dtype=torch.uint8, device=dev) if n else None


class Layer:
    """Inputs of a layer, in surroundings of NaN (pad: elements between the rows)."""

    def __init__(self, dev, B, d_out, d_in, dtype, pad=0, seed=0):
        import torch
        g = _gen(seed, dev)
        self.dev, self.B, self.d_out, self.d_in, self.dtype, self.dt, self.pad = dev, B, d_out, d_in, dtype, _dt(dtype), pad
        self.w = _randn(g, (d_out, d_in), d_in + pad, self.dt, dev, 2 * d_in ** -0.5)
        self.x = _randn(g, (B, d_in), d_in + pad, self.dt, dev)
        self.dy = _randn(g, (B, d_out), d_out + pad, self.dt, dev)
        self.z = _randn(g, (B, d_in), d_in + pad, self.dt, dev, 2.0)
        self.bias = torch.randn(d_out, generator=g, device=dev)
        self.g = g

    def out(self, B, d, dtype):
        return _padded((B, d), d + self.pad, _dt(dtype), self.dev, 7.0)


def _check_fwd(imbd, L, act="none", bias=True, residual=True, keep=True, out=None, in_place=False):
    import torch
    out = out or L.dtype
    y, whole = L.out(L.B, L.d_out, out)
    z, zwhole = L.out(L.B, L.d_out, L.dtype)
    res = _randn(L.g, (L.B, L.d_out), L.d_out + L.pad, _dt(out), L.dev) if residual else None
    r64 = res.double() if residual else 0.0
    if in_place:
        y.copy_(res)
        res = y
    ws = _ws(imbd, 0, L.dtype, L.d_out, L.d_in, L.B, L.dev)
    imbd.linear_fwd(L.w, L.x, y, bias=L.bias if bias else None, act=act, residual=res, z=z if keep else None, ws=ws)
    torch.cuda.synchronize()
    ref, size = L.x.double() @ L.w.double().t(), L.x.double().abs() @ L.w.double().abs().t()
    if bias:
        ref, size = ref + L.bias.double(), size + L.bias.double().abs()
    tol = (L.d_in + 3) * 2 * H * size
    if keep:
        _near(z, ref, tol + STEP[L.dtype] * (ref.abs() + tol), "z")
        assert (zwhole[:, L.d_out:] == 7.0).all()
    v = _value(act, ref)
    tol = 1.13 * tol + _value_err(act, ref)
    total = v + r64
    tol = tol + 2 * H * (v.abs() + total.abs()) + TINY
    _near(y, total, tol + STEP[out] * (total.abs() + tol), "y")
    assert (whole[:, L.d_out:] == 7.0).all()
    return y


def _check_bwd(imbd, L, act="none", residual=True, out=None, which="dw db dx", in_place=False):
    import torch
    out = out or L.dtype
    dw, dw_all = _padded((L.d_out, L.d_in), L.d_in + L.pad, torch.float32, L.dev, 7.0)
    db = torch.full((L.d_out,), 7.0, device=L.dev)
    dx, dx_all = L.out(L.B, L.d_in, out)
    res = _randn(L.g, (L.B, L.d_in), L.d_in + L.pad, _dt(out), L.dev) if residual else None
    r64 = res.double() if residual else 0.0
    if in_place:
        dx.copy_(res)
        res = dx
    imbd.linear_bwd(L.w, L.dy, L.x, dw=dw if "dw" in which else None, db=db if "db" in which else None,
                    dx=dx if "dx" in which else None, act=act, z=L.z if act != "none" else None, residual=res,
                    ws=_ws(imbd, 1, L.dtype, L.d_out, L.d_in, L.B, L.dev))
    torch.cuda.synchronize()
    dy, w, x, z = L.dy.double(), L.w.double(), L.x.double(), L.z.double()
    if "dx" in which:
        v, size = dy @ w, dy.abs() @ w.abs()
        tol = (L.d_out + 2) * 2 * H * size
        d = _slope(act, z)
        ref = v * d + r64
        tol = tol * (d.abs() + SLOPE_ERR[act]) + v.abs() * SLOPE_ERR[act] + 2 * H * ((v * d).abs() + ref.abs()) + TINY
        _near(dx, ref, tol + STEP[out] * (ref.abs() + tol), "dx")
        assert (dx_all[:, L.d_in:] == 7.0).all()
    else:
        assert (dx_all == 7.0).all()
    for name, got, ref, size in (("dw", dw, dy.t() @ x, dy.abs().t() @ x.abs()), ("db", db, dy.sum(0), dy.abs().sum(0))):
        if name in which:
            _near(got, ref, (L.B + 2) * 2 * H * size + H * ref.abs(), name)
        else:
            assert (got == 7.0).all()
    assert (dw_all[:, L.d_in:] == 7.0).all()
    return dw, db, dx


# one row to many, on widths that are and are not whole chunks, tiles and ranges
SHAPES = [(1, 1, 1), (1, 8, 8), (3, 5, 7), (2, 64, 64), (1, 4096, 1024), (5, 4099, 517), (8, 1024, 4096), (16, 200, 1000),
          (17, 512, 2048), (31, 72, 136), (33, 1000, 1001), (64, 4096, 4096), (65, 264, 520), (100, 127, 129), (128, 1024, 256),
          (200, 96, 5000), (255, 257, 255), (256, 1024, 1024), (257, 128, 128), (300, 520, 264), (700, 1000, 784), (1000, 517, 1023),
          (1024, 2048, 512), (2100, 264, 96), (5000, 16, 24), (4097, 136, 72)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,d_out,d_in", SHAPES)
def test_shapes(imbd, dev, B, d_out, d_in, dtype):
    L = Layer(dev, B, d_out, d_in, dtype, seed=B)
    act = ACTS[(B + d_out) % 5]
    _check_fwd(imbd, L, act)
    _check_fwd(imbd, L, "none", bias=False, residual=False, keep=False, out="f32")
    _check_bwd(imbd, L, act)
    _check_bwd(imbd, L, "none", residual=False, out="f32")


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("B,d_out,d_in", [(4, 320, 512), (40, 512, 320), (300, 512, 384), (600, 1024, 768), (90, 77, 91)])
def test_activations(imbd, dev, B, d_out, d_in, act, dtype, out):
    L = Layer(dev, B, d_out, d_in, dtype)
    for bias, residual, keep in ((True, True, True), (False, False, True), (True, False, False), (False, True, False)):
        _check_fwd(imbd, L, act, bias, residual, keep, out)
        _check_bwd(imbd, L, act, residual, out)


@pytest.mark.parametrize("pad", [1, 2, 4, 8, 24])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,d_out,d_in", [(7, 264, 520), (50, 520, 264), (300, 264, 520), (1030, 256, 264), (9, 33, 31)])
def test_pitches(imbd, dev, B, d_out, d_in, dtype, pad):
    L = Layer(dev, B, d_out, d_in, dtype, pad=pad)
    _check_fwd(imbd, L, "gelu_tanh")
    _check_bwd(imbd, L, "silu")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,d_out,d_in", [(7, 264, 520), (50, 520, 264), (300, 264, 520), (1030, 256, 264)])
def test_tensors_that_start_off_a_chunk(imbd, dev, B, d_out, d_in, dtype):
    """One tensor after another begins an element (of 4 bytes: one) into its allocation."""
    import torch
    L = Layer(dev, B, d_out, d_in, dtype)
    for name in ("w", "x", "dy", "z", "bias"):
        old = getattr(L, name)
        flat = torch.full((old.numel() + 1,), float("nan"), dtype=old.dtype, device=dev)
        new = flat[1:].view(old.shape)
        new.copy_(old)
        setattr(L, name, new)
        _check_fwd(imbd, L, "silu")
        _check_bwd(imbd, L, "gelu")
        setattr(L, name, old)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,d_out,d_in", [(3, 128, 256), (100, 256, 128), (400, 256, 256), (30, 61, 67)])
def test_residual_in_place(imbd, dev, B, d_out, d_in, dtype):
    L = Layer(dev, B, d_out, d_in, dtype)
    _check_fwd(imbd, L, "gelu", in_place=True)
    _check_bwd(imbd, L, "relu", in_place=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which", ["dw", "db", "dx", "dw db", "dx db", "dw dx"])
@pytest.mark.parametrize("B,d_out,d_in", [(40, 256, 384), (1500, 264, 136), (70, 33, 45)])
def test_parts_of_the_backward_pass(imbd, dev, B, d_out, d_in, which, dtype):
    _check_bwd(imbd, Layer(dev, B, d_out, d_in, dtype), "silu", which=which)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,d_out,d_in", [(64, 256, 784), (257, 8, 8), (300, 512, 512), (500, 1030, 70), (1000, 517, 1023),
                                          (1024, 512, 560), (2100, 512, 530), (2000, 60, 33), (520, 33, 60), (700, 1501, 1100)])
def test_both_products_of_small_layers(imbd, dev, B, d_out, d_in, dtype):
    """Delta_X and Delta_W in one launch, K whole or in ranges for the one or the other or both; without the one or
    the other of dw and db, the residual in place, rows apart."""
    for pad in (0, 3):
        L = Layer(dev, B, d_out, d_in, dtype, pad=pad, seed=B + d_out)
        _check_bwd(imbd, L, act="gelu", out="f32")
        _check_bwd(imbd, L, act="none", which="db dx", residual=False)
        _check_bwd(imbd, L, act="silu", which="dw dx", in_place=True)


@pytest.mark.parametrize("B,d_out,d_in", [(1, 72, 2048), (3, 264, 2056), (8, 1000, 4096), (16, 2048, 4096), (16, 2040, 4104), (5, 512, 16384)])
def test_few_rows_of_long_sums(imbd, dev, B, d_out, d_in):
    L = Layer(dev, B, d_out, d_in, "bf16", seed=d_in)
    _check_fwd(imbd, L, act="gelu_tanh")
    _check_fwd(imbd, L, keep=False, residual=False, out="f32")


@pytest.mark.parametrize("pad", [0, 3, 4])
@pytest.mark.parametrize("B,d_out,d_in", [(1, 72, 2048), (1, 5, 4), (9, 264, 1028), (16, 8200, 2052), (17, 33, 36), (32, 1000, 1024), (31, 8209, 20),
                                          (4, 8192, 4096)])
def test_few_rows_in_single_precision(imbd, dev, B, d_out, d_in, pad):
    L = Layer(dev, B, d_out, d_in, "f32", pad=pad, seed=d_in)
    _check_fwd(imbd, L, act="gelu")
    _check_fwd(imbd, L, keep=False, bias=False, out="bf16", in_place=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_sums(imbd, dev, dtype):
    """K and B that are cut into ranges, few outputs."""
    _check_fwd(imbd, Layer(dev, 3, 8, 100000, dtype), "relu")
    _check_bwd(imbd, Layer(dev, 40000, 24, 16, dtype), "gelu")
    _check_bwd(imbd, Layer(dev, 33001, 40, 264, dtype), "none")
    _check_bwd(imbd, Layer(dev, 5, 70000, 24, dtype), "gelu_tanh")


@pytest.mark.parametrize("B,d_out,d_in", [(2600, 2571, 2563), (2611, 2576, 2567), (2600, 2573, 2568), (5200, 1301, 2561), (40000, 1031, 129)])
def test_wide_layers_of_odd_widths(imbd, dev, B, d_out, d_in):
    """bf16 rows that are no whole chunks, large enough for the large tiles."""
    L = Layer(dev, B, d_out, d_in, "bf16", pad=B % 3)
    _check_fwd(imbd, L, "gelu_tanh")
    _check_fwd(imbd, L, "none", bias=False, residual=False, keep=False, out="f32")
    _check_bwd(imbd, L, "silu")
    _check_bwd(imbd, L, "none", residual=False, out="f32", which="dx db")
    _check_bwd(imbd, L, "gelu", in_place=True, which="dx")


def test_no_rows(imbd, dev):
    import torch
    for dtype in ("bf16", "f32"):
        L = Layer(dev, 0, 64, 32, dtype)
        imbd.linear_fwd(L.w, L.x, torch.empty(0, 64, dtype=L.dt, device=dev))
        dw, db = torch.full((64, 32), 7.0, device=dev), torch.full((64,), 7.0, device=dev)
        imbd.linear_bwd(L.w, L.dy, L.x, dw=dw, db=db, dx=torch.empty(0, 32, dtype=L.dt, device=dev))
        assert (dw == 0).all() and (db == 0).all()
        imbd.act_bwd(L.dy, L.dy, L.dy, "silu")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_act_bwd(imbd, dev, act, dtype):
    import torch
    for B, d, pad in ((1, 1, 0), (3, 7, 2), (64, 1000, 0), (300, 517, 5), (2, 100001, 1)):
        g = _gen(B, dev)
        dy, z = _randn(g, (B, d), d + pad, _dt(dtype), dev), _randn(g, (B, d), d + pad, _dt(dtype), dev, 3.0)
        dz, whole = _padded((B, d), d + pad, _dt(dtype), dev, 7.0)
        imbd.act_bwd(dy, z, dz, act)
        ref = dy.double() * _slope(act, z.double())
        tol = dy.double().abs() * SLOPE_ERR[act] + H * ref.abs() + TINY
        _near(dz, ref, tol + STEP[dtype] * (ref.abs() + tol), act)
        assert (whole[:, d:] == 7.0).all()
        for place in (dy, z):
            a, b = dy.clone(), z.clone()
            t = a if place is dy else b
            imbd.act_bwd(a, b, t, act)
            assert torch.equal(t, dz)


@pytest.mark.parametrize("act", ACTS)
def test_far_values(imbd, dev, act):
    """Activations and derivatives where exponentials leave the range of fp32, through a layer of one weight."""
    import torch
    z = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 5, -5, 13, -13, 40, -40, 90, -90, 700, -700, 1e10, -1e10, 1e19, -1e19, 1e30, -1e30],
                     device=dev)[:, None].contiguous()
    w, y = torch.ones(1, 1, device=dev), torch.empty_like(z)
    imbd.linear_fwd(w, z, y, act=act)
    ref = _value(act, z.double())
    _near(y, ref, _value_err(act, z.double()).nan_to_num(0, 0, 0) + 2 * H * ref.abs() + 2.0 ** -110, "y")
    dz = torch.empty_like(z)
    imbd.act_bwd(w.expand(20, 1).contiguous(), z, dz, act)
    _near(dz, _slope(act, z.double()), torch.full_like(ref, max(SLOPE_ERR[act], 2 * H)), "dz")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,d_out,d_in", [(4, 256, 512), (60, 256, 512), (400, 512, 256), (40, 67, 61)])
def test_not_a_number_stays_in_its_row(imbd, dev, B, d_out, d_in, dtype):
    """NaN and infinities reach the outputs that they belong to, and no others."""
    import torch
    for act in ACTS:
        L = Layer(dev, B, d_out, d_in, dtype)
        L.x[1, d_in - 1] = float("nan")
        L.x[3, 0] = float("inf")
        y = torch.full((B, d_out), 7.0, dtype=L.dt, device=dev)
        imbd.linear_fwd(L.w, L.x, y, act=act, ws=_ws(imbd, 0, dtype, d_out, d_in, B, dev))
        assert y[1].isnan().all() and not y[[0, 2]].isnan().any() and (not y[4:].isnan().any())
        dw, db = torch.empty(d_out, d_in, device=dev), torch.empty(d_out, device=dev)
        L.x[3, 0] = 1.0
        imbd.linear_bwd(L.w, L.dy, L.x, dw=dw, db=db, ws=_ws(imbd, 1, dtype, d_out, d_in, B, dev))
        assert dw[:, d_in - 1].isnan().all() and not dw[:, :d_in - 1].isnan().any() and not db.isnan().any()


def test_backward_against_differences(imbd, dev):
    """Of sum(c * y) by x, w and b through two layers, the lower one's activation in the upper one's backward pass."""
    import torch
    B, d0, d1, d2 = 3, 5, 6, 4
    g = _gen(0, dev)

    def r(*s):
        return torch.randn(*s, generator=g, device=dev)

    for act in ACTS[2:]:
        p = dict(x=r(B, d0), w1=r(d1, d0), b1=r(d1), w2=r(d2, d1), b2=r(d2), res=r(B, d2))
        c = r(B, d2)

        def f(q):
            h, y = torch.empty(B, d1, device=dev), torch.empty(B, d2, device=dev)
            imbd.linear_fwd(q["w1"], q["x"], h, bias=q["b1"], act=act)
            imbd.linear_fwd(q["w2"], h, y, bias=q["b2"], residual=q["res"])
            return (c * y).double().sum().item()

        h, z = torch.empty(B, d1, device=dev), torch.empty(B, d1, device=dev)
        imbd.linear_fwd(p["w1"], p["x"], h, bias=p["b1"], act=act, z=z)
        grad = {k: torch.empty_like(v) for k, v in p.items()}
        dz = torch.empty(B, d1, device=dev)
        imbd.linear_bwd(p["w2"], c, h, dw=grad["w2"], db=grad["b2"], dx=dz, act=act, z=z)
        imbd.linear_bwd(p["w1"], dz, p["x"], dw=grad["w1"], db=grad["b1"], dx=grad["x"])
        grad["res"] = c  # (a residual's gradient is that of the output)
        step = 2.0 ** -6
        for k, v in p.items():
            for i in range(v.numel()):
                q = [dict(p), dict(p)]
                for s, o in zip((step, -step), q):
                    o[k] = v.clone()
                    o[k].view(-1)[i] += s
                slope = (f(q[0]) - f(q[1])) / (2 * step)
                # third derivatives of the activations are under 2, weights and inputs mostly under 3: step^2 / 6 * 2 * 27 * 27 sums to
                # under 0.06 here; the differences' own rounding is under 1e-3
                assert abs(slope - grad[k].view(-1)[i].item()) <= 0.06, (act, k, i)


def test_repeats_on_another_stream_and_in_a_graph(imbd, dev):
    """The same bits on every run, on a stream of the caller's and replayed from a graph after the inputs changed; two layers share
    one workspace."""
    import torch
    for B, d_out, d_in, dtype in ((8, 1024, 2048, "bf16"), (60, 1024, 2048, "bf16"), (700, 512, 512, "bf16"), (50, 99, 3001, "f32")):
        L = Layer(dev, B, d_out, d_in, dtype)
        o = dict(y=torch.zeros(B, d_out, dtype=L.dt, device=dev), z=torch.zeros(B, d_out, dtype=L.dt, device=dev),
                 dw=torch.zeros(d_out, d_in, device=dev), db=torch.zeros(d_out, device=dev),
                 dx=torch.zeros(B, d_in, dtype=L.dt, device=dev))
        code = imbd.dtype_code(L.dt)
        n = max(imbd.linear_workspace_bytes(k, code, d_out, d_in, B) for k in (0, 1))
        ws = torch.full((max(n, 8),), 255, dtype=torch.uint8, device=dev)

        def call():
            imbd.linear_fwd(L.w, L.x, o["y"], bias=L.bias, act="gelu", z=o["z"], ws=ws)
            imbd.linear_bwd(L.w, o["y"], L.x, dw=o["dw"], db=o["db"], dx=o["dx"], act="silu", z=L.z, ws=ws)

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
        for _ in range(2):
            graph.replay()
            again = take()
            assert all(torch.equal(first[k], again[k]) and torch.equal(first[k], other[k]) for k in first)
        L.x.normal_(generator=_gen(5, dev))
        call()
        eager = take()
        graph.replay()
        again = take()
        assert all(torch.equal(eager[k], again[k]) for k in eager) and not torch.equal(eager["y"], first["y"])


def test_tensors_elsewhere_are_refused(imbd, dev):
    import torch
    w, x, y = torch.zeros(8, 4, device=dev), torch.zeros(3, 4, device=dev), torch.zeros(3, 8, device=dev)
    for call in (lambda: imbd.linear_fwd(w.cpu(), x, y), lambda: imbd.linear_fwd(w, x.cpu(), y),
                 lambda: imbd.linear_fwd(w, x, y, ws=torch.zeros(8)), lambda: imbd.linear_fwd(w, x, y.t().contiguous().t()),
                 lambda: imbd.linear_bwd(w, y, x.cpu(), dw=w)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(imbd.ImbdError):
        imbd.linear_fwd(w, x[:1].expand(3, 4), y)
