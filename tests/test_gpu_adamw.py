"""AdamW over many tensors against its formulas in 64 bits, and its 8-bit state against their definition.

A 32-bit state is off by at most the roundings of its formula: m and v three each (two products, a sum; v one
more for the square), so 4 * 2^-24 of the terms' sizes. The update lr * m_hat / (sqrt(v_hat) + eps) has m and v
(4 each), a square root and a division within one unit, four products and sums: under 16 * 2^-24 of it, and
the weight itself two roundings."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-6)
SIZES = [1, 3, 4, 255, 256, 257, 1000, 4095, 4096, 4097, 70001, 1 << 18]


def _tensors(dev, sizes, bits, grad, seed, lp=True, shift=0):
    """Tensors as slices of larger buffers, `shift` elements from their start, in surroundings of 5."""
    import torch
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        def new(dtype, v, m=n):
            if dtype.itemsize == 1:
                whole = torch.full((m + shift + 8,), 5, dtype=torch.uint8, device=dev).view(dtype)
            else:
                whole = torch.full((m + shift + 8,), 5.0, dtype=dtype, device=dev)
            part = whole[shift:shift + m]
            part.copy_(v)
            return part, whole
        t, whole = {}, {}
        scale = 10.0 ** -(i % 4)
        r = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
        t["w"], whole["w"] = new(torch.float32, r(n))
        t["grad"], whole["grad"] = new(torch.bfloat16 if grad == "bf16" else torch.float32, r(n) * scale)
        if lp:
            t["w_lp"], whole["w_lp"] = new(torch.bfloat16, r(n))
        if bits == 32:
            t["m"], whole["m"] = new(torch.float32, r(n) * scale)
            t["v"], whole["v"] = new(torch.float32, (r(n) * scale) ** 2)
        else:
            nb = (n + 255) // 256
            mc = torch.randint(0, 0x7F, (n,), generator=g, device=dev).to(torch.uint8)  # no NaN code
            mc |= (torch.randint(0, 2, (n,), generator=g, device=dev) * 128).to(torch.uint8)
            vc = torch.randint(0, 0x7C, (n,), generator=g, device=dev).to(torch.uint8)
            vc[(vc > 0) & (vc < 4)] = 4
            t["m"], whole["m"] = new(torch.float8_e4m3fn, mc.view(torch.float8_e4m3fn))
            t["v"], whole["v"] = new(torch.float8_e5m2, vc.view(torch.float8_e5m2))
            t["m_scale"], whole["m_scale"] = new(torch.float32, r(nb).abs() * scale / 448, nb)
            t["v_scale"], whole["v_scale"] = new(torch.float32, r(nb).abs() * scale ** 2 / 57344, nb)
        t["decay"] = 0.0 if i % 3 == 0 else 0.1
        out.append((t, whole))
    return out


def _values(t, key):
    """The state as 64-bit values."""
    n = t["w"].numel()
    v = t[key].double()
    if t["m"].dtype.itemsize == 1:
        v = v * t[key + "_scale"].double().repeat_interleave(256)[:n]
    return v


def _ref(t, step, gs=1.0, lr=0.0, beta1=0.0, beta2=0.0, eps=0.0):
    """(w, m, v, size of m's terms) after one step, before any rounding of the state."""
    g = t["grad"].double() * float(np.float32(gs))
    w, m, v = t["w"].double(), _values(t, "m"), _values(t, "v")
    m2 = beta1 * m + (1 - beta1) * g
    size = beta1 * m.abs() + (1 - beta1) * g.abs()
    v2 = beta2 * v + (1 - beta2) * g * g
    den = (v2 / (1 - beta2 ** step)).sqrt() + eps
    upd = lr / (1 - beta1 ** step) * m2 / den
    return w * (1 - lr * t["decay"]) - upd, m2, v2, size, lr / (1 - beta1 ** step) * size / den


def _dither21(n, step):
    i = np.arange(n, dtype=np.uint64)
    low = np.uint64(0xFFFFFFFF)
    h = (i + np.uint64(step) * np.uint64(0x9E3779B9)) & low
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x7FEB352D)) & low
    h = ((h ^ (h >> np.uint64(15))) * np.uint64(0x846CA68B)) & low
    return ((h ^ (h >> np.uint64(16))) >> np.uint64(11)).astype(np.int64)


def _check_step(imbd, pairs, step, gs=1.0, step_arg=None):
    import torch
    before = [{k: (v.clone() if hasattr(v, "clone") else v) for k, v in t.items()} for t, _ in pairs]
    plan = imbd.AdamW([t for t, _ in pairs])
    imbd.adamw_step(plan, step=step if step_arg is None else step_arg, grad_scale=gs, **HYPER)
    torch.cuda.synchronize()
    e = 2.0 ** -24
    for (t, whole), old in zip(pairs, before):
        n = t["w"].numel()
        w, m, v, msize, usize = _ref(old, step, gs, **HYPER)
        err = (t["w"].double() - w).abs()
        tol = 16 * e * usize + 3 * e * (w.abs() + old["w"].double().abs())
        assert (err <= tol).all(), (n, (err / tol).max().item())
        if "w_lp" in t:
            assert torch.equal(t["w_lp"], t["w"].to(torch.bfloat16))
        if t["m"].dtype.itemsize != 1:
            assert ((t["m"].double() - m).abs() <= 4 * e * msize).all()
            assert ((t["v"].double() - v).abs() <= 6 * e * v).all()
        else:
            nb = (n + 255) // 256
            pad = torch.zeros(nb * 256, dtype=torch.float64, device=m.device)
            pad[:n] = m.abs()
            ms = pad.view(nb, 256).amax(1)
            pad[:n] = v
            vs = pad.view(nb, 256).amax(1)
            # the scales: the block's largest value (as above; its size may exceed it by cancellation) times a constant
            pad[:n] = msize
            slack = pad.view(nb, 256).amax(1)
            assert ((t["m_scale"].double() * 448 - ms).abs() <= 8 * e * slack).all()
            assert ((t["v_scale"].double() * 57344 - vs).abs() <= 10 * e * vs).all()
            sm = t["m_scale"].double().repeat_interleave(256)[:n]
            sv = t["v_scale"].double().repeat_interleave(256)[:n]
            # m: to nearest e4m3: half a step, 2^-4 of a normal value, half of 2^-9 below
            q, r = t["m"].double(), m / torch.where(sm > 0, sm, torch.ones_like(sm))
            assert ((q - r).abs() <= torch.maximum(r.abs(), q.abs()) * 2.0 ** -4 + 2.0 ** -10 + 16 * e * 448).all()
            # v: one of the two e5m2 neighbours, the upper one where the dropped 21 bits and the dither carry
            r = (v / torch.where(sv > 0, sv, torch.ones_like(sv))).cpu().numpy()
            d = _dither21(n, step)
            q = t["v"].float().cpu().numpy().astype(np.float64)
            with np.errstate(divide="ignore"):
                ulp = 2.0 ** (np.floor(np.log2(np.where(r > 0, r, 1.0))) - 2)
            want = np.floor(r / ulp + d / 2.0 ** 21) * ulp
            want = np.where(r > 0, np.clip(want, 2.0 ** -14, 57344.0), 0.0)
            differ = q != want
            # where r is within its own rounding of a border (16 * 2^-24 relative of steps of 1/4 and finer: at most
            # 8 * 16 * 2^-24 of the elements), the code may be the neighbour
            assert differ.sum() <= max(2, 1e-3 * n), (n, differ.sum())
            assert (np.abs(q - want) <= 1.01 * ulp + 2.0 ** -14)[differ].all()
        for k, b in whole.items():
            s = t[k].storage_offset()
            out = torch.cat([b[:s].view(torch.uint8), b[s + t[k].numel():].view(torch.uint8)])
            full = torch.full_like(b.view(torch.uint8), 5) if b.dtype.itemsize == 1 else torch.full_like(b, 5.0).view(torch.uint8)
            assert torch.equal(out, full[:out.numel()]), k


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_many_sizes(imbd, dev, bits, grad, shift):
    pairs = _tensors(dev, SIZES, bits, grad, seed=bits + shift, shift=shift)
    _check_step(imbd, pairs, 1)
    _check_step(imbd, pairs, 2, gs=0.125)
    _check_step(imbd, pairs, 1000)


@pytest.mark.parametrize("bits", [32, 8])
def test_mixed_set_and_empty_tensors(imbd, dev, bits):
    """32- and 8-bit states, both gradient types, with and without a copy, and tensors of no elements, in one plan."""
    pairs = (_tensors(dev, [5, 0, 3000], 32, "f32", 1) + _tensors(dev, [700, 9000], 8, "bf16", 2, lp=False) +
             _tensors(dev, [0, 8192], bits, "bf16", 3, shift=2))
    _check_step(imbd, pairs, 7)


def test_first_step_from_zero_state(imbd, dev):
    """Zero state, zero gradients in places: no NaN, and w moves by lr * sign(g) in the first step (eps aside)."""
    import torch
    for bits in (32, 8):
        (t, whole), = _tensors(dev, [5000], bits, "f32", 4)
        t["m"].view(torch.uint8).zero_()
        t["v"].view(torch.uint8).zero_()
        t["grad"][:600] = 0.0   # two whole blocks and a part
        t["decay"] = 0.0
        w0 = t["w"].clone()
        _check_step(imbd, [(t, whole)], 1)
        assert torch.equal(t["w"][:600], w0[:600])
        assert not t["m"].float()[:600].any() and not t["v"].float()[:512].any()


def test_a_second_moment_moves_at_a_rate_below_its_step(imbd, dev):
    """v decays by 1% a step, under half a step of its format: after 100 steps without gradients a tensor's mean of v
    is 0.99^100 of what it was, within the dither's spread. (The blocks' largest element keeps its gradient, so the
    scales stay.)"""
    import torch
    n, nb = 256 * 200, 200
    z = lambda dt: torch.zeros(n, dtype=torch.uint8, device=dev).view(dt)  # noqa: E731
    t = {"w": torch.zeros(n, device=dev), "grad": torch.zeros(n, device=dev), "m": z(torch.float8_e4m3fn),
         "v": z(torch.float8_e5m2), "m_scale": torch.zeros(nb, device=dev), "v_scale": torch.zeros(nb, device=dev)}
    t["grad"][::256] = 1.0
    t["v"].copy_(torch.full((n,), 4096.0, device=dev))
    t["v"][::256] = 57344.0
    t["v_scale"].fill_(1.0 / 57344)
    plan = imbd.AdamW([t])
    for s in range(1, 101):
        imbd.adamw_step(plan, lr=0.0, beta1=0.9, beta2=0.99, step=s)
    v = (t["v"].float().view(nb, 256) * t["v_scale"][:, None])[:, 1:]
    want = 4096.0 / 57344 * 0.99 ** 100
    # a step's rounding moves an element by at most a quarter of itself, with a mean of zero: over 100 steps with
    # 51000 elements, each at most 0.25 * sqrt(100 * 0.04) of the mean (a move happens in 4% of steps), a mean over
    # them within 6 * 0.5 / sqrt(51000) = 1.4%; pseudo-random bits shared by blocks of one index: none here (one tensor)
    assert abs(v.mean().item() / want - 1) < 0.03, v.mean().item() / want


def test_non_finite_gradients(imbd, dev):
    """A NaN or an infinity stays in its element (32 bits) or its block of 256 (8 bits)."""
    import torch
    for bits in (32, 8):
        (t, _), = _tensors(dev, [1024], bits, "f32", 5)
        (c, _), = _tensors(dev, [1024], bits, "f32", 5)
        t["grad"][300] = float("nan")
        t["grad"][700] = float("inf")
        for x in (t, c):
            imbd.adamw_step(imbd.AdamW([x]), step=3, **HYPER)
        keep = torch.ones(1024, dtype=torch.bool, device=dev)
        keep[[300, 700]] = False
        assert torch.equal(t["w"][keep], c["w"][keep])
        assert torch.isnan(t["w"][300]) and not torch.isfinite(t["w"][700])
        if bits == 8:
            keep[256:768] = False
        for k in ("m", "v"):
            a, b = _values(t, k), _values(c, k)
            assert torch.equal(a[keep], b[keep])
            assert not torch.isfinite(a[300]) and not torch.isfinite(a[700])


def test_a_first_moment_that_decays_to_nothing(imbd, dev):
    """Without gradients m shrinks by beta1 a step until its scale is a few of the smallest fp32 numbers (u = 2^-149),
    where the scale is rounded by up to a third. Against the exact m: half a code's step (16 scales), what lies past
    448 scales, and the fp32 roundings of the code times its scale and of the product with beta1 (u / 2 each)."""
    import torch
    nb, u = 64, 2.0 ** -149
    t = dict(w=torch.randn(256 * nb, device=dev), grad=torch.zeros(256 * nb, device=dev),
             m=torch.full((256 * nb,), 0x7E, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn),
             v=torch.full((256 * nb,), 0x7B, dtype=torch.uint8, device=dev).view(torch.float8_e5m2),
             m_scale=(torch.arange(1, nb + 1, device=dev).double() * u).float(),
             v_scale=torch.full((nb,), 1e-6, device=dev), decay=0.0)
    t["m"].view(torch.uint8)[1::2] |= 0x80
    plan, w = imbd.AdamW([t]), t["w"].clone()
    for step in range(900, 960):
        exact = _values(t, "m") * HYPER["beta1"]
        imbd.adamw_step(plan, step=step, **HYPER)
        got, s = _values(t, "m"), t["m_scale"].double().repeat_interleave(256)
        assert torch.isfinite(got).all()
        bound = 16 * s + (exact.abs() - 448 * s).clamp(min=0) + u
        bound = torch.where(s == 0, exact.abs() + u, bound)
        assert ((got - exact).abs() <= bound).all(), step
    assert torch.equal(t["w"], w)  # (steps of 1e-40)


def test_step_from_device_and_graph(imbd, dev):
    """The step's number in device memory: the bits of the same number as an argument, and a replayed graph follows
    the counter."""
    import torch
    for bits in (32, 8):
        a = [t for t, _ in _tensors(dev, [5000, 300], bits, "bf16", 6)]
        b = [t for t, _ in _tensors(dev, [5000, 300], bits, "bf16", 6)]
        pa, pb = imbd.AdamW(a), imbd.AdamW(b)
        count = torch.ones(1, dtype=torch.int32, device=dev)
        imbd.adamw_step(pa, step=1, **HYPER)
        imbd.adamw_step(pb, step=count, **HYPER)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            count.add_(1)
            imbd.adamw_step(pb, step=count, **HYPER)
        for s in range(2, 7):
            graph.replay()
            imbd.adamw_step(pa, step=s, **HYPER)
            torch.cuda.synchronize()
            for x, y in zip(a, b):
                for k in x:
                    if k != "decay":
                        assert torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)), (bits, s, k)


def test_same_bits_again_and_beside_others(imbd, dev):
    """A tensor's result does not depend on what else is in the plan."""
    import torch
    for bits in (32, 8):
        many = [t for t, _ in _tensors(dev, SIZES, bits, "f32", 8)]
        alone = [t for t, _ in _tensors(dev, SIZES, bits, "f32", 8)]
        imbd.adamw_step(imbd.AdamW(many), step=5, **HYPER)
        for t in alone:
            imbd.adamw_step(imbd.AdamW([t]), step=5, **HYPER)
        torch.cuda.synchronize()
        for x, y in zip(many, alone):
            for k in x:
                if k != "decay":
                    assert torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8))


@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_same_bits_in_a_set_past_the_caches(imbd, dev, grad):
    """A set of more than 512 MB reads and writes past the caches: the bits stay."""
    import torch
    n = 20_000_000
    z = lambda: torch.zeros(n, device=dev)  # noqa: E731
    big = {"w": z(), "w_lp": z().to(torch.bfloat16), "grad": z(), "m": z(), "v": z()}
    for bits in (32, 8):
        pairs = _tensors(dev, SIZES, bits, grad, seed=8)
        alone = [t for t, _ in _tensors(dev, SIZES, bits, grad, seed=8)]
        imbd.adamw_step(imbd.AdamW([big] + [t for t, _ in pairs]), step=5, **HYPER)
        imbd.adamw_step(imbd.AdamW(alone), step=5, **HYPER)
        torch.cuda.synchronize()
        for (x, whole), y in zip(pairs, alone):
            for k in x:
                if k != "decay":
                    assert torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)), k
    assert not big["w"].any() and not big["v"].any()


def test_refusals(imbd, dev):
    import torch
    (t, _), = _tensors(dev, [512], 32, "f32", 9)
    plan = imbd.AdamW([t])
    with pytest.raises(imbd.ImbdError):
        imbd.adamw_step(plan, lr=1e-3, step=0)
    with pytest.raises(imbd.ImbdError):
        imbd.adamw_step(plan, lr=float("nan"))
    with pytest.raises(imbd.ImbdError):
        imbd.adamw_step(plan, lr=1e-3, beta2=1.0)
    with pytest.raises(TypeError):
        imbd.adamw_step(plan, lr=1e-3, step=torch.ones(1, dtype=torch.int64, device=dev))
    with pytest.raises(TypeError):
        imbd.AdamW([{**t, "grad": t["grad"].half()}])
    with pytest.raises(TypeError):
        imbd.AdamW([{**t, "v": t["v"].to(torch.float8_e5m2)}])
    with pytest.raises(ValueError):
        imbd.AdamW([{**t, "m": t["m"][:-1]}])
    with pytest.raises(ValueError):
        imbd.AdamW([{**t, "grad": t["grad"].cpu()}])
    with pytest.raises(ValueError):
        imbd.AdamW([{**t, "w": t["w"][::2], "m": t["m"][::2], "v": t["v"][::2], "grad": t["grad"][::2], "w_lp": None}])
    with pytest.raises(imbd.ImbdError):
        imbd.AdamW([{**t, "decay": -1.0}])
    imbd.adamw_step(imbd.AdamW([]), lr=1e-3)
    torch.cuda.synchronize()


class _Beside:
    """The binding, its plans with one more tensor."""

    def __init__(self, imbd, other):
        self.imbd, self.other, self.plan = imbd, other, None

    def AdamW(self, tensors):
        self.plan = self.imbd.AdamW([self.other, *tensors])
        return self.plan

    def adamw_step(self, *args, **kw):
        return self.imbd.adamw_step(*args, **kw)


# the plan's flags of a tensor, and what adamw_write_plan compares with 336 MiB: every array of the set once
GRAD_BF16, STATE8, VECTOR, STREAM = 1, 2, 4, 8
RECORD, FLAGS_AT = 72, 68


def _footprint(t):
    each = sum(t[k].element_size() for k in ("w", "grad", "m", "v"))
    return t["w"].numel() * (each + (2 if t.get("w_lp") is not None else 0))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_steps_past_the_caches(imbd, dev, bits, grad):
    """Every form of the update that loads and stores past the caches against the formulas in 64 bits, and its bits
    against those of a small set. (A test of the set's size and of the plan's flags: these forms have run.)"""
    import torch
    n = 40_000_000
    big = {k: torch.zeros(n, device=dev, dtype=dt) for k, dt in
           (("w", torch.float32), ("w_lp", torch.bfloat16), ("grad", torch.float32), ("m", torch.float32), ("v", torch.float32))}
    assert _footprint(big) > 600 << 20
    beside = _Beside(imbd, big)
    pairs = _tensors(dev, SIZES, bits, grad, seed=18)
    alone = [t for t, _ in _tensors(dev, SIZES, bits, grad, seed=18)]
    assert sum(_footprint(t) for t in alone) < 64 << 20
    small = imbd.AdamW(alone)
    for step in (1, 2, 1000):
        _check_step(beside, pairs, step)
        imbd.adamw_step(small, step=step, **HYPER)
    flags = [int.from_bytes(bytes(beside.plan.plan[i * RECORD + FLAGS_AT:][:4].tolist()), "little") for i in range(len(SIZES) + 1)]
    want = VECTOR | STREAM | (STATE8 if bits == 8 else 0) | (GRAD_BF16 if grad == "bf16" else 0)
    assert flags == [VECTOR | STREAM] + [want] * len(SIZES)
    assert not int.from_bytes(bytes(small.plan[FLAGS_AT:][:4].tolist()), "little") & STREAM
    for (x, _), y in zip(pairs, alone):
        for k in x:
            if k != "decay":
                assert torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)), k
    assert not big["w"].any() and not big["m"].any() and not big["v"].any() and not big["w_lp"].any()


def test_a_large_tensor_past_the_caches(imbd, dev):
    """A tensor that is itself past the caches, to its last element: 8 million against the formulas, the others still."""
    import torch
    n = 36_000_003
    big = {k: torch.zeros(n, device=dev, dtype=dt) for k, dt in
           (("w", torch.float32), ("grad", torch.float32), ("m", torch.float32), ("v", torch.float32))}
    assert _footprint(big) > 336 << 20
    (t, _), = _tensors(dev, [8_000_003], 32, "f32", 19)
    tail = {k: v[n - 8_000_003:] for k, v in big.items()}
    for k in tail:
        tail[k].copy_(t[k])
    old = {k: v.clone() for k, v in tail.items()}
    imbd.adamw_step(imbd.AdamW([big]), step=4, **HYPER)
    w, m, v, msize, usize = _ref({**old, "decay": 0.0}, 4, **HYPER)
    e = 2.0 ** -24
    assert ((tail["w"].double() - w).abs() <= 16 * e * usize + 3 * e * (w.abs() + old["w"].double().abs())).all()
    assert ((tail["m"].double() - m).abs() <= 4 * e * msize).all() and ((tail["v"].double() - v).abs() <= 6 * e * v).all()
    assert not any(big[k][:n - 8_000_003].any() for k in big)
