"""The expert layer's operators against plain implementations in 64 bits.

Tolerances are bounds, not fits. A product's sum of K terms in fp32 is off by at most
(K + 2) * 2^-23 * sum |terms| (one unit in the last place for each product and addition, whatever their
order), and storing it as bf16 adds half a step, 2^-8 of the value; both are applied element by element."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a rounding step, relative


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed, dev):
    import torch
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return g


def _padded(shape, ld, dtype, dev, fill=float("nan")):
    """(view, whole buffer): rows of `shape` at a pitch of ld elements, `fill` in what lies between them."""
    import torch
    whole = torch.full((*shape[:-1], ld), fill, dtype=dtype, device=dev)
    return whole[..., :shape[-1]], whole


def _randn(g, shape, ld, dtype, dev, scale=1.0):
    import torch
    v, _ = _padded(shape, ld, dtype, dev)
    v.copy_(torch.randn(shape, generator=g, device=dev) * scale)
    return v


class Layer:
    """An expert layer's inputs from the number of slots of each expert, in surroundings of NaN."""

    def __init__(self, dev, counts, d_out, d_in, dtype, gather=False, spare=0, pad=0, seed=0, n_x=None):
        import torch
        g = _gen(seed, dev)
        self.counts, self.E, self.dev = counts, len(counts), dev
        self.d_out, self.d_in, self.dtype, self.dt = d_out, d_in, dtype, _dt(dtype)
        self.used = sum(counts)
        self.n = self.used + spare
        self.offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device=dev)
        self.w = _randn(g, (self.E, d_out, d_in), d_in + pad, self.dt, dev, d_in ** -0.5)
        self.bias = torch.randn(self.E, d_out, generator=g, device=dev)
        self.n_x = n_x if n_x is not None else (max(1, self.n // 2) if gather else self.n)
        self.x = _randn(g, (self.n_x, d_in), d_in + pad, self.dt, dev)
        self.dy = _randn(g, (self.n, d_out), d_out + pad, self.dt, dev)
        self.rows = torch.randint(0, self.n_x, (self.n,), generator=g, device=dev, dtype=torch.int32) if gather else None
        self.pad = pad

    def xs(self):
        """x in expert order, in 64 bits; an index outside x is a row of zeros."""
        import torch
        if self.rows is None:
            return self.x.double()
        r = self.rows.long()
        ok = (r >= 0) & (r < self.n_x)
        x = self.x.double()[r.clamp(0, max(self.n_x - 1, 0))]
        return torch.where(ok[:, None], x, torch.zeros_like(x))

    def each(self):
        a = 0
        for e, c in enumerate(self.counts):
            yield e, slice(a, a + c)
            a += c


def _close(got, ref, size, K, out, what):
    """|got - ref| within (K + 2) 2^-23 size plus half a step of the output's type."""
    err = (got.double() - ref).abs()
    tol = (K + 2) * 2.0 ** -23 * size + STEP[out] * (ref.abs() + (K + 2) * 2.0 ** -23 * size)
    bad = ~(err <= tol)
    assert not bad.any(), (what, bad.sum().item(), bad.numel(), (err / tol.clamp(min=1e-300)).max().item())


def _check_fwd(imbd, L, relu=False, bias=True, out=None):
    import torch
    out = out or L.dtype
    y, whole = _padded((L.n, L.d_out), L.d_out + L.pad, _dt(out), L.dev, 7.0)
    imbd.expert_fwd(L.w, L.x, L.offsets, y, bias=L.bias if bias else None, relu=relu, rows=L.rows)
    torch.cuda.synchronize()
    xs = L.xs()
    for e, s in L.each():
        w = L.w[e].double()
        ref, size = xs[s] @ w.t(), xs[s].abs() @ w.abs().t()
        if bias:
            ref, size = ref + L.bias[e].double(), size + L.bias[e].double().abs()
        if relu:
            ref = ref.clamp(min=0)
        _close(y[s], ref, size, L.d_in + 1, out, f"y of expert {e}")
    assert (y[L.used:] == 7.0).all()
    assert (whole[:, L.d_out:] == 7.0).all()


def _check_bwd(imbd, L, mask=False, out=None, which="dw db dx", call=True):
    import torch
    out = out or L.dtype
    dw, dw_all = _padded((L.E, L.d_out, L.d_in), L.d_in + L.pad, torch.float32, L.dev, 7.0)
    db = torch.full((L.E, L.d_out), 7.0, device=L.dev)
    dx, dx_all = _padded((L.n, L.d_in), L.d_in + L.pad, _dt(out), L.dev, 7.0)
    imbd.expert_bwd(L.w, L.dy, L.x, L.offsets, dw=dw if "dw" in which else None, db=db if "db" in which else None,
                    dx=dx if "dx" in which else None, rows=L.rows, mask_relu=mask)
    torch.cuda.synchronize()
    xs = L.xs()
    for e, s in L.each():
        dy, w, x, K = L.dy[s].double(), L.w[e].double(), xs[s], L.counts[e]
        if "dx" in which:
            ref, size = dy @ w, dy.abs() @ w.abs()
            if mask:
                ref, size = ref * (x > 0), size * (x > 0)
            _close(dx[s], ref, size, L.d_out, out, f"dx of expert {e}")
        if "dw" in which:
            _close(dw[e], dy.t() @ x, dy.abs().t() @ x.abs(), K, "f32", f"dw of expert {e}")
        if "db" in which:
            _close(db[e], dy.sum(0), dy.abs().sum(0), K, "f32", f"db of expert {e}")
    if "dx" in which:
        assert (dx[L.used:] == 7.0).all() and (dx_all[:, L.d_in:] == 7.0).all()
    else:
        assert (dx_all == 7.0).all()
    if "dw" not in which:
        assert (dw_all == 7.0).all()
    assert (dw_all[..., L.d_in:] == 7.0).all()
    return dw, db, dx


COUNTS = {
    "one": [1],
    "ragged": [3, 0, 65, 64, 1, 0, 129, 40],
    "empty": [0, 0, 0],
    "edges": [0, 127, 128, 255, 256, 257, 1],
    "one_takes_all": [0, 0, 700, 0],
    "many": [(7 * e) % 23 for e in range(150)],
}


# ---------------------------------------------------------------------------- products
@pytest.mark.parametrize("counts", list(COUNTS))
@pytest.mark.parametrize("d_out,d_in,dtype", [(72, 136, "bf16"), (101, 77, "bf16"), (67, 45, "f32"), (1, 1, "bf16"),
                                              (8, 3, "f32"), (64, 128, "f32")])
@pytest.mark.parametrize("gather", [False, True])
def test_products_small(imbd, dev, counts, d_out, d_in, dtype, gather):
    L = Layer(dev, COUNTS[counts], d_out, d_in, dtype, gather=gather, spare=5, seed=len(counts) + d_out)
    _check_fwd(imbd, L, relu=gather)
    _check_bwd(imbd, L, mask=not gather)


@pytest.mark.parametrize("counts", ["ragged", "edges", "one_takes_all"])
@pytest.mark.parametrize("d_out,d_in,pad", [(512, 256, 0), (520, 264, 8), (136, 1032, 16), (1000, 328, 3), (384, 512, 24),
                                            (128, 64, 0), (2048, 96, 8)])
@pytest.mark.parametrize("gather", [False, True])
def test_products_bf16_layers(imbd, dev, counts, d_out, d_in, pad, gather):
    """Widths of one to several large tiles, with pitches that are whole 16-byte chunks and one that is not."""
    L = Layer(dev, COUNTS[counts], d_out, d_in, "bf16", gather=gather, spare=3, pad=pad, seed=d_out + pad)
    _check_fwd(imbd, L, relu=True)
    _check_bwd(imbd, L, mask=True)


@pytest.mark.parametrize("wide,K", [(3832, 72), (3840, 200), (3832, 328), (3840, 64), (3832, 8)])
@pytest.mark.parametrize("counts", [[2500, 1600], [1, 4090, 9]])
@pytest.mark.parametrize("gather,out", [(False, "bf16"), (True, "bf16"), (True, "f32")])
def test_products_on_tiles_of_256_rows(imbd, dev, wide, K, counts, gather, out):
    """Sizes whose tiles of 256 rows are one round of the CUs and those of 128 two, which is where the larger tile is
    taken; K from less than one slab to several, even and odd numbers of them, whole and cut."""
    L = Layer(dev, counts, wide, K, "bf16", gather=gather, spare=2, pad=8, seed=K)
    _check_fwd(imbd, L, relu=gather, out=out)
    L = Layer(dev, counts, K, wide, "bf16", gather=gather, spare=2, pad=8, seed=K)
    _check_bwd(imbd, L, mask=True, out=out)


@pytest.mark.parametrize("dtype,d_out,d_in", [("bf16", 256, 512), ("bf16", 264, 99), ("f32", 66, 70)])
@pytest.mark.parametrize("gather", [False, True])
def test_bias_gradient_without_x(imbd, dev, dtype, d_out, d_in, gather):
    """db alone needs no x; dw of slots whose rows do not exist (an x of no rows) is zero."""
    import torch
    L = Layer(dev, [5, 0, 130, 300], d_out, d_in, dtype, gather=gather, seed=4)
    want = _check_bwd(imbd, L, which="db")[1]
    db = torch.full((L.E, d_out), 7.0, device=dev)
    imbd.expert_bwd(L.w, L.dy, None, L.offsets, db=db, rows=L.rows)
    assert torch.equal(db, want)
    if gather:
        dw = torch.full((L.E, d_out, d_in), 7.0, device=dev)
        imbd.expert_bwd(L.w, L.dy, L.x[:0], L.offsets, dw=dw, db=db, rows=L.rows)
        assert not dw.any() and torch.equal(db, want)
    # dx alone without a mask needs no x either
    dx, ref = (torch.zeros(L.n, d_in, dtype=L.dt, device=dev) for _ in range(2))
    imbd.expert_bwd(L.w, L.dy, None, L.offsets, dx=dx)
    imbd.expert_bwd(L.w, L.dy, L.x, L.offsets, dx=ref, rows=L.rows)
    assert torch.equal(dx, ref)


def test_long_rows_and_many_slots(imbd, dev):
    """Offsets past 32 bits of bytes in every operand: x gathered from the end of more than 4 GiB (the kernel for any
    size), rows in expert order past 4 GiB (the large tiles, whose windows move), and their gradients."""
    import torch
    n_x, d = 70000, 32768  # 4.6 GB of bf16
    big = torch.zeros(n_x, d, dtype=torch.bfloat16, device=dev)
    g = _gen(1, dev)
    big[-3:] = torch.randn(3, d, generator=g, device=dev)
    w = (torch.randn(2, 64, d, generator=g, device=dev) * d ** -0.5).to(torch.bfloat16)
    bias = torch.randn(2, 64, generator=g, device=dev)
    rows = torch.tensor([n_x - 1, n_x - 3, 5, n_x - 2] * 30, dtype=torch.int32, device=dev)
    off = torch.tensor([0, 50, 120], dtype=torch.int32, device=dev)
    y = torch.zeros(120, 64, device=dev)
    imbd.expert_fwd(w, big, off, y, bias=bias, rows=rows)
    for e, s in ((0, slice(0, 50)), (1, slice(50, 120))):
        x = big[rows[s].long()].double()
        _close(y[s], x @ w[e].double().t() + bias[e].double(), x.abs() @ w[e].double().abs().t() + bias[e].double().abs(),
               d + 1, "f32", "gathered")
    # in expert order: the last expert owns the last rows
    off = torch.tensor([0, n_x - 3, n_x], dtype=torch.int32, device=dev)
    y = torch.zeros(n_x, 64, dtype=torch.bfloat16, device=dev)
    imbd.expert_fwd(w, big, off, y, bias=bias)
    x = big[-3:].double()
    _close(y[-3:], x @ w[1].double().t() + bias[1].double(), x.abs() @ w[1].double().abs().t() + bias[1].double().abs(), d + 1,
           "bf16", "in order")
    assert torch.equal(y[:-3], bias[0].to(torch.bfloat16).expand(n_x - 3, 64))
    dy = torch.zeros(n_x, 64, dtype=torch.bfloat16, device=dev)
    dy[-3:] = torch.randn(3, 64, generator=g, device=dev)
    dw, db = torch.empty(2, 64, d, device=dev), torch.empty(2, 64, device=dev)
    dx = torch.full((n_x, d), 3.0, dtype=torch.bfloat16, device=dev)
    imbd.expert_bwd(w, dy, big, off, dw=dw, db=db, dx=dx)
    c = dy[-3:].double()
    _close(dw[1], c.t() @ x, c.abs().t() @ x.abs(), 3, "f32", "dw")
    _close(db[1], c.sum(0), c.abs().sum(0), 3, "f32", "db")
    _close(dx[-3:], c @ w[1].double(), c.abs() @ w[1].double().abs(), 64, "bf16", "dx")
    assert not dw[0].any() and not dx[:-3].any()


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts", ["ragged", "edges"])
def test_products_output_types(imbd, dev, dtype, out, counts):
    L = Layer(dev, COUNTS[counts], 264, 200, dtype, gather=True, seed=3)
    _check_fwd(imbd, L, bias=False, out=out)
    _check_bwd(imbd, L, out=out)


@pytest.mark.parametrize("which", ["dw", "db", "dx", "dw db", "dx db"])
@pytest.mark.parametrize("dtype,d", [("bf16", 256), ("bf16", 99), ("f32", 70)])
def test_backward_parts(imbd, dev, which, dtype, d):
    """Each output by itself has the bits that it has beside the others."""
    import torch
    L = Layer(dev, [5, 0, 130, 300], d, d + 8, dtype, gather=True, seed=4)
    one = _check_bwd(imbd, L, which=which, mask=True)
    all3 = _check_bwd(imbd, L, mask=True)
    for name, a, b in zip(("dw", "db", "dx"), one, all3):
        if name in which.split():
            assert torch.equal(a, b), name


@pytest.mark.parametrize("counts", [[1], [2, 0, 1], [8, 8], [1] * 16, [0, 16, 3, 1, 0, 33]])
@pytest.mark.parametrize("d_out,d_in,dtype", [(512, 1024, "bf16"), (1024, 520, "bf16"), (4096, 4096, "bf16"),
                                              (1000, 1024, "bf16"), (264, 1000, "bf16"), (257, 1023, "bf16"),
                                              (300, 500, "f32")])
@pytest.mark.parametrize("gather", [False, True])
def test_single_tokens(imbd, dev, counts, d_out, d_in, dtype, gather):
    """The forward product for a handful of rows, as decoding makes it."""
    L = Layer(dev, counts, d_out, d_in, dtype, gather=gather, seed=sum(counts) + d_in)
    _check_fwd(imbd, L, relu=gather, bias=not gather)


@pytest.mark.parametrize("dtype,d_out,d_in", [("bf16", 256, 512), ("bf16", 130, 70), ("f32", 66, 70)])
def test_rows_outside_x_read_as_zeros(imbd, dev, dtype, d_out, d_in):
    import torch
    L = Layer(dev, [4, 200, 0, 30], d_out, d_in, dtype, gather=True, spare=2, seed=5)
    bad = torch.tensor([-1, L.n_x, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=dev)
    L.rows[::7] = bad[torch.arange(len(L.rows[::7]), device=dev) % 4]
    _check_fwd(imbd, L)
    _check_bwd(imbd, L, mask=True)


@pytest.mark.parametrize("dtype,d", [("bf16", 256), ("bf16", 101), ("f32", 40)])
def test_offsets_are_clamped(imbd, dev, dtype, d):
    """Offsets past the rows, or falling ones, reach nothing outside the arrays; the experts whose offsets are
    sound get their results."""
    import torch
    L = Layer(dev, [100, 60], d, d + 8, dtype, seed=6)
    L.offsets = torch.tensor([0, 100, 100000], dtype=torch.int32, device=dev)
    _check_fwd(imbd, L)
    _check_bwd(imbd, L)
    L = Layer(dev, [0, 0, 160], d, d + 8, dtype, seed=6)
    L.offsets = torch.tensor([-5, 0, -7, 160], dtype=torch.int32, device=dev)  # expert 1: none; 2: all
    _check_fwd(imbd, L)
    _check_bwd(imbd, L)
    L = Layer(dev, [0, 0], d, d + 8, dtype, spare=160, seed=6)
    L.offsets = torch.tensor([2 ** 31 - 1, 5, -2 ** 31], dtype=torch.int32, device=dev)
    _check_fwd(imbd, L)
    _check_bwd(imbd, L)


def test_no_rows(imbd, dev):
    """No rows at all: the weights' and biases' gradients are zeros."""
    import torch
    L = Layer(dev, [0, 0], 64, 64, "bf16", seed=7)
    dw, db = torch.ones(2, 64, 64, device=dev), torch.ones(2, 64, device=dev)
    dx = torch.empty(0, 64, dtype=torch.bfloat16, device=dev)
    imbd.expert_bwd(L.w, L.dy, L.x, L.offsets, dw=dw, db=db, dx=dx)
    imbd.expert_fwd(L.w, L.x, L.offsets, torch.empty(0, 64, dtype=torch.bfloat16, device=dev))
    torch.cuda.synchronize()
    assert not dw.any() and not db.any()
    # every slot of x missing
    L = Layer(dev, [3, 2], 64, 64, "bf16", gather=True, n_x=1, seed=8)
    L.x, L.n_x = L.x[:0], 0
    y = torch.empty(5, 64, dtype=torch.bfloat16, device=dev)
    imbd.expert_fwd(L.w, L.x, L.offsets, y, bias=L.bias, rows=L.rows)
    assert torch.equal(y, L.bias.to(torch.bfloat16)[[0, 0, 0, 1, 1]])


@pytest.mark.parametrize("dtype,d_out,d_in,n", [("bf16", 264, 512, 300), ("bf16", 99, 45, 40), ("bf16", 512, 256, 5),
                                                ("f32", 70, 40, 90)])
def test_infinities_and_nans_stay_in_their_rows(imbd, dev, dtype, d_out, d_in, n):
    """What is not finite in one slot's input reaches that slot's results and its expert's gradients alone."""
    import torch
    L = Layer(dev, [n, n], d_out, d_in, dtype, seed=9)
    clean = Layer(dev, [n, n], d_out, d_in, dtype, seed=9)
    L.x[n - 1, 0] = float("nan")
    L.x[2, d_in - 1] = float("inf")
    outs = []
    for l in (L, clean):
        y = torch.zeros(l.n, d_out, dtype=l.dt, device=dev)
        imbd.expert_fwd(l.w, l.x, l.offsets, y, relu=True)
        dw, db = torch.zeros(2, d_out, d_in, device=dev), torch.zeros(2, d_out, device=dev)
        dx = torch.zeros(l.n, d_in, dtype=l.dt, device=dev)
        imbd.expert_bwd(l.w, l.dy, l.x, l.offsets, dw=dw, db=db, dx=dx)
        outs.append((y, dw, db, dx))
    (y, dw, db, dx), (yc, dwc, dbc, dxc) = outs
    keep = [i for i in range(2 * n) if i not in (2, n - 1)]
    assert torch.equal(y[keep], yc[keep]) and torch.isnan(y[n - 1]).all()
    assert torch.equal(dw[1], dwc[1]) and torch.equal(db, dbc) and torch.equal(dx, dxc)
    assert torch.isnan(dw[0, :, 0]).all() and torch.equal(dw[0, :, 1:d_in - 1], dwc[0, :, 1:d_in - 1])


@pytest.mark.parametrize("dtype,d_out,d_in", [("bf16", 512, 256), ("bf16", 101, 77), ("f32", 64, 64)])
def test_same_bits_again(imbd, dev, dtype, d_out, d_in):
    import torch
    L = Layer(dev, COUNTS["edges"], d_out, d_in, dtype, gather=True, seed=10)
    got = []
    for _ in range(3):
        y = torch.empty(L.n, d_out, dtype=L.dt, device=dev)
        imbd.expert_fwd(L.w, L.x, L.offsets, y, bias=L.bias, rows=L.rows)
        got.append([y] + [t.clone() for t in _check_bwd(imbd, L)])
    for g in got[1:]:
        for a, b in zip(g, got[0]):
            assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))


def test_gradients_against_differences(imbd, dev):
    """d(sum(y * c)) along a direction of w, b and x, by central differences in fp32 of a product that is linear in
    each of them (so the difference quotient has no error but the sums' rounding)."""
    import torch
    L = Layer(dev, [5, 0, 12, 33], 40, 24, "f32", gather=True, seed=11)
    g = _gen(12, dev)

    def f(w, b, x):
        y = torch.zeros(L.n, L.d_out, device=dev)
        imbd.expert_fwd(w, x, L.offsets, y, bias=b, rows=L.rows)
        return (y.double() * L.dy.double()).sum().item()

    dw, db, dx = _check_bwd(imbd, L)
    slots = torch.argsort(L.rows.long(), stable=True)
    dxt = torch.zeros(L.n_x, L.d_in, dtype=torch.float64, device=dev).index_add_(0, L.rows.long(), dx.double())
    assert slots.numel() == L.n
    for name, v, grad in (("w", L.w, dw), ("bias", L.bias, db), ("x", L.x, dxt)):
        u = torch.randn(v.shape, generator=g, device=dev)
        args = {"w": L.w, "b": L.bias, "x": L.x}
        key = {"w": "w", "bias": "b", "x": "x"}[name]
        hi, lo = f(**{**args, key: v + u}), f(**{**args, key: v - u})
        want = (grad.double() * u.double()).sum().item()
        # each y is off by at most (24 + 3) 2^-23 of its terms' sizes (about 40 here), times |dy| over 2000 outputs
        assert abs((hi - lo) / 2 - want) < 2000 * 27 * 2.0 ** -23 * 40 * 3, (name, hi, lo, want)


# ------------------------------------------------------------------------------ router
def _route_ref(z, k, renorm):
    """The router in 64 bits: (gates, experts, offsets, rows, slots, probabilities)."""
    z = z.astype(np.float64)
    T, E = z.shape
    rank = np.where(np.isnan(z), np.inf, z)
    # NaN above +inf: two stable sorts, by value and then NaN first
    order = np.argsort(-rank, axis=1, kind="stable")
    isn = np.take_along_axis(np.isnan(z), order, 1)
    order = np.take_along_axis(order, np.argsort(~isn, axis=1, kind="stable"), 1)
    experts = order[:, :k]
    picked = np.take_along_axis(z, experts, 1)
    dead = picked == -np.inf
    with np.errstate(invalid="ignore", over="ignore"):
        peak = np.where(np.isneginf(z.max(1, keepdims=True)), 0.0, z.max(1, keepdims=True))
        p = np.exp(z - peak)
        pp = np.where(dead, 0.0, np.exp(picked - peak))
        tot = pp.sum(1, keepdims=True) if renorm else p.sum(1, keepdims=True)
        gates = np.where(dead, 0.0, pp / np.where(tot == 0, 1.0, tot))
        prob = p / np.where(tot == 0, 1.0, tot)
    experts = np.where(dead, -1, experts)
    t, j = np.nonzero(experts >= 0)
    e = experts[t, j]
    o = np.lexsort((j, t, e))
    slots = np.full((T, k), -1)
    slots[t[o], j[o]] = np.arange(len(o))
    return gates, experts, np.searchsorted(e[o], np.arange(E + 1)), t[o], slots, prob


def _route(imbd, z, k, renorm, dev):
    import torch
    T, E = z.shape
    i32 = dict(dtype=torch.int32, device=dev)
    gates = torch.full((T, k), 9.0, device=dev)
    experts, offsets = torch.full((T, k), 9, **i32), torch.full((E + 1,), 9, **i32)
    rows, slots = torch.full((T * k,), -9, **i32), torch.full((T, k), 9, **i32)
    ws = torch.full((imbd.expert_route_workspace_bytes(T, E, k),), 0xFF, dtype=torch.uint8, device=dev)
    imbd.expert_route(z, gates, experts, offsets, rows, slots, ws, renorm=renorm)
    torch.cuda.synchronize()
    return gates, experts, offsets, rows, slots


def _check_route(imbd, z, k, renorm, dev):
    got = _route(imbd, z, k, renorm, dev)
    gates, experts, offsets, rows, slots = (t.cpu().numpy() for t in got)
    rg, re, ro, rr, rs, prob = _route_ref(z.cpu().numpy(), k, renorm)
    assert np.array_equal(experts, re)
    assert np.array_equal(offsets, ro)
    assert np.array_equal(rows[:len(rr)], rr) and (rows[len(rr):] == -9).all()
    assert np.array_equal(slots, rs)
    assert np.array_equal(np.isnan(gates), np.isnan(rg))
    # exp of a difference d rounded to 2^-24 |d| (at most 2^-24 * 110 relative in the result, smaller ones are
    # zero in fp32), a library exp within 2 ulp, a sum of E of them and a division: under (|d| + E + 8) 2^-23
    with np.errstate(invalid="ignore"):
        err = np.abs(gates - rg)
        ok = np.isnan(rg) | (err <= rg * (110 + z.shape[1] + 8) * 2.0 ** -23 + 2.0 ** -126)
    assert ok.all(), (err[~ok][:5], rg[~ok][:5])
    return got, (rg, re, prob)


@pytest.mark.parametrize("T", [1, 2, 7, 127, 128, 129, 1000, 5003])
@pytest.mark.parametrize("E,k", [(1, 1), (2, 1), (3, 3), (8, 2), (10, 4), (64, 8), (65, 6), (128, 2), (200, 9), (256, 8),
                                 (257, 1), (500, 16), (512, 16)])
@pytest.mark.parametrize("renorm", [False, True])
def test_route(imbd, dev, T, E, k, renorm):
    import torch
    g = _gen(T * 1000 + E, dev)
    z = _padded((T, E), E + T % 3, torch.float32, dev)[0]
    z.copy_(torch.randn(T, E, generator=g, device=dev) * 3)
    _check_route(imbd, z, k, renorm, dev)


@pytest.mark.parametrize("T,E,k", [(40, 64, 8), (300, 10, 4), (700, 130, 5)])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_ties_and_masks(imbd, dev, T, E, k, renorm):
    """Many equal logits (the lowest experts win), zeros of both signs, whole and partial masks, the type's
    lowest and largest values, NaN and infinity."""
    import torch
    g = _gen(T + E, dev)
    z = torch.randint(-2, 3, (T, E), generator=g, device=dev).float()
    z[1] = 0.0
    z[1, 1::2] = -0.0
    z[2] = -float("inf")
    z[3, 2:] = -float("inf")
    z[4] = torch.finfo(torch.float32).min
    z[5, 1:] = torch.finfo(torch.float32).min
    z[6] = torch.finfo(torch.float32).max
    z[7] = -float("inf")
    z[7, E - 1] = torch.finfo(torch.float32).min
    z[8, E // 2] = float("inf")
    z[9, 3] = float("nan")
    z[10, 1] = z[10, E - 1] = float("nan")
    z[11] = float("nan")
    z[12:14] = 1e-40
    z[12, 4] = 2e-40
    z[15:20] = -float("inf")
    _check_route(imbd, z, k, renorm, dev)


def test_route_everything_masked_and_no_tokens(imbd, dev):
    import torch
    z = torch.full((300, 6), -float("inf"), device=dev)
    (gates, experts, offsets, rows, slots), _ = _check_route(imbd, z, 2, True, dev)
    assert not offsets.any() and (experts == -1).all() and not gates.any()
    _, _, offsets, _, _ = _route(imbd, torch.empty(0, 6, device=dev), 2, True, dev)
    assert not offsets.any()
    imbd.expert_route_bwd(None, torch.empty(0, 2, device=dev), torch.empty(0, 2, dtype=torch.int32, device=dev),
                          torch.empty(0, 2, device=dev), torch.empty(0, 6, device=dev))


def test_route_many_tokens(imbd, dev):
    """More tokens than the table of workgroups has rows of 128."""
    import torch
    g = _gen(1, dev)
    _check_route(imbd, torch.randn(70001, 16, generator=g, device=dev), 2, True, dev)
    z = torch.zeros(40000, 4, device=dev)  # all on the first expert
    z[:, 0] = 1.0
    _check_route(imbd, z, 1, False, dev)


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (37, 10, 4), (500, 64, 8), (100, 130, 2), (64, 300, 16), (9, 512, 1)])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_bwd(imbd, dev, T, E, k, renorm):
    import torch
    g = _gen(T + E + k, dev)
    z = torch.randn(T, E, generator=g, device=dev) * 2
    z[T // 2] = -float("inf")
    if T > 3:
        z[3, 1:] = -float("inf")
    (gates, experts, _, _, _), (rg, re, prob) = _check_route(imbd, z, k, renorm, dev)
    dg = torch.randn(T, k, generator=g, device=dev)
    dz, whole = _padded((T, E), E + 5, torch.float32, dev, 7.0)
    imbd.expert_route_bwd(None if renorm else z, gates, experts, dg, dz, renorm=renorm)
    torch.cuda.synchronize()
    d = dg.cpu().numpy().astype(np.float64)
    inner = (rg * d).sum(1, keepdims=True)
    ref = np.zeros((T, E))
    t, j = np.nonzero(re >= 0)
    np.add.at(ref, (t, re[t, j]), (rg * (d - (inner if renorm else 0)))[t, j])
    if not renorm:
        ref -= np.where(np.isnan(prob), 0, prob) * inner
    # each factor within (110 + E + 8) 2^-23 (the gates), their products and sums of k + 2 terms
    size = np.abs(rg * d).sum(1, keepdims=True) + np.abs(d).max(1, keepdims=True) * np.abs(rg).max(1, keepdims=True)
    err = np.abs(dz.cpu().numpy() - ref)
    assert (err <= 2 * (110 + E + k + 10) * 2.0 ** -23 * size + 1e-37).all(), err.max()
    assert (whole[:, E:] == 7.0).all()


def test_route_gradient_against_differences(imbd, dev):
    import torch
    g = _gen(5, dev)
    T, E, k = 20, 12, 3
    z = torch.randn(T, E, generator=g, device=dev)
    c = torch.randn(T, k, generator=g, device=dev)
    u = torch.randn(T, E, generator=g, device=dev)
    h = 2.0 ** -10
    for renorm in (False, True):
        (gates, experts, *_), _ = _check_route(imbd, z, k, renorm, dev)
        dz = torch.zeros(T, E, device=dev)
        imbd.expert_route_bwd(z, gates, experts, c, dz, renorm=renorm)
        f = []
        for s in (h, -h):
            gs, es, *_ = _route(imbd, z + s * u, k, renorm, dev)
            same = (es == experts).all(1)
            f.append(((gs.double() * c.double()).sum(1), same))
        rows = f[0][1] & f[1][1]
        assert rows.sum() >= T - 4
        got = (f[0][0] - f[1][0])[rows] / (2 * h)
        want = (dz.double() * u.double()).sum(1)[rows]
        # third derivative of a softmax along u: at most 6 |u|^3 |c| (|u| < 4, |c| < 4), times h^2 / 6; rounding of
        # the gates 130 * 2^-23 over h
        assert ((got - want).abs() < 4 ** 4 * h * h + 3 * 4 * 130 * 2.0 ** -23 / h).all()


def test_route_bwd_of_a_repeated_expert(imbd, dev):
    """Pairs of the caller's own: an expert named twice takes both gradients, -1 none."""
    import torch
    experts = torch.tensor([[1, 1], [2, -1]], dtype=torch.int32, device=dev)
    gates = torch.tensor([[0.5, 0.25], [0.5, 0.5]], device=dev)
    dg = torch.tensor([[2.0, 4.0], [8.0, 16.0]], device=dev)
    dz = torch.full((2, 3), 9.0, device=dev)
    imbd.expert_route_bwd(None, gates, experts, dg, dz, renorm=True)
    # inner: 0.5*2 + 0.25*4 = 2; 0.5*8 = 4
    assert torch.equal(dz, torch.tensor([[0.0, 0.5 * 0 + 0.25 * 2, 0.0], [0.0, 0.0, 0.5 * 4]], device=dev))


# ----------------------------------------------------------------------------- combine
@pytest.mark.parametrize("T,k,d", [(1, 1, 1), (1, 4, 4096), (5, 3, 77), (130, 2, 512), (33, 16, 264), (64, 1, 1000),
                                   (300, 8, 40)])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("pad", [0, 8, 3])
def test_combine(imbd, dev, T, k, d, dtype, out, pad):
    import torch
    g = _gen(T + k + d, dev)
    n = T * k + 3
    slots = torch.randperm(T * k, generator=g, device=dev).to(torch.int32).view(T, k).contiguous()
    gates = torch.randn(T, k, generator=g, device=dev)
    ys = _randn(g, (n, d), d + pad, _dt(dtype), dev)
    dy = _randn(g, (T, d), d + pad, _dt(dtype), dev)
    if T > 4:  # pairs without a slot; their gates do not matter
        slots[1] = -1
        gates[1] = float("nan")
        slots[2, 0] = n
        slots[3, k - 1] = -2 ** 31
    ok = ((slots >= 0) & (slots < n)).double()
    at = slots.long().clamp(0, n - 1)
    v = torch.where(ok[..., None] > 0, ys.double()[at], torch.zeros((), dtype=torch.float64, device=dev))
    gd = torch.where(ok > 0, gates.double(), torch.zeros((), dtype=torch.float64, device=dev))
    for gt in (gates, None):
        y, whole = _padded((T, d), d + pad, _dt(out), dev, 7.0)
        imbd.expert_combine(ys, slots, y, gates=gt)
        wt = (gd if gt is not None else ok)[..., None]
        _close(y, (v * wt).sum(1), (v * wt).abs().sum(1), k, out, "y")
        assert (whole[:, d:] == 7.0).all()
    if out != dtype:
        return
    for with_gates in (True, False):
        dys, whole = _padded((n, d), d + pad, _dt(dtype), dev, 7.0)
        dg = torch.full((T, k), 7.0, device=dev) if with_gates else None
        imbd.expert_combine_bwd(dy, ys if with_gates else None, slots, gates, dys, dg)
        torch.cuda.synchronize()
        want = torch.full((n, d), 7.0, dtype=torch.float64, device=dev)
        real = ok.bool()
        want[slots.long()[real]] = (gd[..., None] * dy.double()[:, None, :])[real]
        _close(dys, want, want.abs(), 1, dtype, "dys")
        assert (whole[:, d:] == 7.0).all()
        if with_gates:
            dyv = dy.double()[:, None, :]
            _close(dg, (v * dyv).sum(2), (v * dyv).abs().sum(2), d, "f32", "dgates")


# ------------------------------------------------------------------- together, as used
def _step(imbd, p, b, x, target):
    """One training step of a two-layer expert network on buffers b: router, experts, loss gradient of
    sum (y - target)^2 / 2, backward, AdamW on every weight."""
    imbd.expert_route(b["z"], b["gates"], b["experts"], b["offsets"], b["rows"], b["slots"], b["ws"])
    imbd.expert_fwd(p["w1"], x, b["offsets"], b["h"], bias=p["b1"], relu=True, rows=b["rows"])
    imbd.expert_fwd(p["w2"], b["h"], b["offsets"], b["ys"], bias=p["b2"])
    imbd.expert_combine(b["ys"], b["slots"], b["y"], gates=b["gates"])
    b["dy"].copy_(b["y"] - target)
    imbd.expert_combine_bwd(b["dy"], b["ys"], b["slots"], b["gates"], b["dys"], b["dgates"])
    imbd.expert_bwd(p["w2"], b["dys"], b["h"], b["offsets"], dw=b["dw2"], db=b["db2"], dx=b["dh"], mask_relu=True)
    imbd.expert_bwd(p["w1"], b["dh"], x, b["offsets"], dw=b["dw1"], db=b["db1"], dx=b["dxs"], rows=b["rows"])
    imbd.expert_combine(b["dxs"], b["slots"], b["dx"])
    imbd.expert_route_bwd(b["z"], b["gates"], b["experts"], b["dgates"], b["dz"])


def _network(imbd, dev, T, E, k, d, dh, dtype, seed, pad_tokens=0):
    import torch
    g = _gen(seed, dev)
    dt = _dt(dtype)
    f32 = dict(device=dev)
    i32 = dict(dtype=torch.int32, device=dev)
    m = {"w1": torch.randn(E, dh, d, generator=g, device=dev) * d ** -0.5,
         "w2": torch.randn(E, d, dh, generator=g, device=dev) * dh ** -0.5,
         "b1": torch.randn(E, dh, generator=g, device=dev) * 0.1, "b2": torch.randn(E, d, generator=g, device=dev) * 0.1}
    p = {"w1": m["w1"].to(dt), "w2": m["w2"].to(dt), "b1": m["b1"], "b2": m["b2"]}
    x = torch.randn(T, d, generator=g, device=dev).to(dt)
    target = torch.randn(T, d, generator=g, device=dev).to(dt)
    n = T * k
    b = {"z": torch.randn(T, E, generator=g, device=dev), "gates": torch.zeros(T, k, **f32),
         "experts": torch.zeros(T, k, **i32), "offsets": torch.zeros(E + 1, **i32), "rows": torch.zeros(n, **i32),
         "slots": torch.zeros(T, k, **i32),
         "ws": torch.zeros(imbd.expert_route_workspace_bytes(T, E, k), dtype=torch.uint8, device=dev),
         "h": torch.zeros(n, dh, dtype=dt, **f32), "ys": torch.zeros(n, d, dtype=dt, **f32),
         "y": torch.zeros(T, d, dtype=dt, **f32), "dy": torch.zeros(T, d, dtype=dt, **f32),
         "dys": torch.zeros(n, d, dtype=dt, **f32), "dgates": torch.zeros(T, k, **f32),
         "dw2": torch.zeros(E, d, dh, **f32), "db2": torch.zeros(E, d, **f32), "dh": torch.zeros(n, dh, dtype=dt, **f32),
         "dw1": torch.zeros(E, dh, d, **f32), "db1": torch.zeros(E, dh, **f32), "dxs": torch.zeros(n, d, dtype=dt, **f32),
         "dx": torch.zeros(T, d, dtype=dt, **f32), "dz": torch.zeros(T, E, **f32)}
    if pad_tokens:
        b["z"][T - pad_tokens:] = -float("inf")
    return m, p, b, x, target


def _network_ref(p, b, x, target, k):
    """The same network by automatic differentiation in 64 bits on the CPU."""
    import torch
    f64 = {n: t.double().cpu().requires_grad_() for n, t in
           {**p, "x": x, "z": b["z"]}.items()}
    z, xx = f64["z"], f64["x"]
    experts = b["experts"].long().cpu()
    on = experts >= 0
    picked = torch.gather(z, 1, experts.clamp(min=0))
    picked = torch.where(on, picked, torch.full_like(picked, -float("inf")))
    gates = torch.softmax(torch.where(on.any(1, keepdim=True), picked, torch.zeros_like(picked)), 1) * on
    y = torch.zeros_like(xx)
    for e in range(z.shape[1]):
        for j in range(k):
            t = torch.nonzero(experts[:, j] == e)[:, 0]
            if len(t):
                h = torch.relu(xx[t] @ f64["w1"][e].t() + f64["b1"][e])
                o = h @ f64["w2"][e].t() + f64["b2"][e]
                y = y.index_add(0, t, gates[t, j:j + 1] * o)
    live = on.any(1).double()[:, None]  # (a token without experts has y = 0: no gradient passes)
    (0.5 * ((y - target.double().cpu()) ** 2) * live).sum().backward()
    return {n: t.grad for n, t in f64.items()}, y.detach()


@pytest.mark.parametrize("T,E,k,d,dh,dtype,pad", [(50, 5, 2, 24, 40, "f32", 0), (200, 8, 2, 128, 256, "f32", 7),
                                                  (300, 6, 3, 256, 512, "bf16", 11), (90, 16, 4, 72, 56, "bf16", 0)])
def test_a_network_of_experts(imbd, dev, T, E, k, d, dh, dtype, pad):
    """Routing, both layers, the combination, and the backward pass to every weight, the input and the logits."""
    m, p, b, x, target = _network(imbd, dev, T, E, k, d, dh, dtype, T, pad)
    _step(imbd, p, b, x, target)
    ref, y = _network_ref(p, b, x, target, k)
    # normwise: fp32 sums of at most T*k + d + dh terms; bf16 stores h, ys, y, dy, dys, dh, dxs, dx, each at 2^-8,
    # with cancellation in the sums over k and over y - target (a factor of 4), 8 in a row at most
    tol = 8 * 4 * 2.0 ** -8 if dtype == "bf16" else 4 * (T * k + d + dh) * 2.0 ** -23
    got = {"w1": b["dw1"], "w2": b["dw2"], "b1": b["db1"], "b2": b["db2"], "x": b["dx"], "z": b["dz"]}
    assert (b["y"].double().cpu() - y).norm() <= tol * y.norm()
    for name, gr in got.items():
        e = (gr.double().cpu() - ref[name]).norm() / ref[name].norm()
        assert e <= tol, (name, e.item())


def test_captured_and_replayed(imbd, dev):
    """The whole step in a graph, replayed on new inputs between eager steps: every replay has the eager bits."""
    import torch
    for dtype, d, dh, T in (("bf16", 256, 512, 300), ("f32", 40, 24, 60)):
        m, p, b, x, target = _network(imbd, dev, T, 6, 2, d, dh, dtype, 3, 4)
        _, _, eager, _, _ = _network(imbd, dev, T, 6, 2, d, dh, dtype, 3, 4)
        _step(imbd, p, b, x, target)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            _step(imbd, p, b, x, target)
        torch.cuda.current_stream().wait_stream(s)
        with torch.cuda.graph(graph):
            _step(imbd, p, b, x, target)
        g = _gen(4, dev)
        for i in range(4):
            x.copy_(torch.randn(x.shape, generator=g, device=dev))
            z = torch.randn(T, 6, generator=g, device=dev)
            for buf in (b, eager):
                buf["z"].copy_(z)
            graph.replay()
            _step(imbd, p, eager, x, target)
            torch.cuda.synchronize()
            for name in b:
                if name == "ws":
                    continue
                used = int(eager["offsets"][-1])
                a, c = b[name], eager[name]
                if name in ("rows", "h", "ys", "dys", "dh", "dxs"):
                    a, c = a[:used], c[:used]
                assert torch.equal(a, c), (i, name)


def test_on_another_stream(imbd, dev):
    """Calls go to the stream they are given, or to the current one."""
    import torch
    L = Layer(dev, [100, 200], 256, 128, "bf16", seed=1)
    y, y2 = (torch.zeros(L.n, 256, dtype=torch.bfloat16, device=dev) for _ in range(2))
    imbd.expert_fwd(L.w, L.x, L.offsets, y)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=dev)
    with torch.cuda.stream(s):
        for _ in range(10):
            big = big @ big * 1e-3
        L2x = L.x * 1.0
        imbd.expert_fwd(L.w, L2x, L.offsets, y2)  # has to wait for the product above it
    s.synchronize()
    assert torch.equal(y, y2)
    y2.zero_()
    torch.cuda.synchronize()
    imbd.expert_fwd(L.w, L.x, L.offsets, y2, stream=s)
    s.synchronize()
    assert torch.equal(y, y2)


def test_refusals(imbd, dev):
    """What does not fit together is refused before anything is launched."""
    import torch
    L = Layer(dev, [3, 5], 64, 32, "bf16", gather=True, seed=1)
    y = torch.full((8, 64), 7.0, dtype=torch.bfloat16, device=dev)
    for bad in (dict(w=L.w[:, :, :-1]), dict(w=L.w[:1]), dict(x=L.x.float()), dict(x=L.x.cpu()), dict(offsets=L.offsets.long()),
                dict(offsets=L.offsets[:-1]), dict(rows=L.rows[:-1]), dict(rows=L.rows.long()), dict(bias=L.bias.half()),
                dict(bias=L.bias[:, :-1]), dict(y=y[:, ::2]), dict(y=y.half()), dict(w=L.w.transpose(1, 2)), dict(w=L.w.cpu()),
                dict(x=L.x[:1].expand(L.n_x, 32)), dict(w=L.w[:1].expand(2, 64, 32)), dict(rows=None)):
        a = {**dict(w=L.w, x=L.x, offsets=L.offsets, y=y, bias=L.bias, rows=L.rows), **bad}
        with pytest.raises((ValueError, TypeError, imbd.ImbdError)):
            imbd.expert_fwd(**a)
    dw, db = torch.full((2, 64, 32), 7.0, device=dev), torch.full((2, 64), 7.0, device=dev)
    for bad in (dict(dw=dw[:1]), dict(dw=dw.bfloat16()), dict(db=db[:, 1:]), dict(dy=L.dy[:, :-1]), dict(x=None),
                dict(dw=None, db=None), dict(dx=torch.empty(8, 31, device=dev)), dict(dx=torch.empty(8, 32, device=dev).double())):
        a = {**dict(w=L.w, dy=L.dy, x=L.x, offsets=L.offsets, dw=dw, db=db, rows=L.rows), **bad}
        with pytest.raises((ValueError, TypeError, imbd.ImbdError)):
            imbd.expert_bwd(**a)
    z = torch.zeros(1000, 8, device=dev)
    f, i = lambda *s: torch.zeros(*s, device=dev), lambda *s: torch.zeros(*s, dtype=torch.int32, device=dev)  # noqa: E731
    ok = dict(logits=z, gates=f(1000, 2), experts=i(1000, 2), offsets=i(9), rows=i(2000), slots=i(1000, 2),
              ws=torch.zeros(imbd.expert_route_workspace_bytes(1000, 8, 2), dtype=torch.uint8, device=dev))
    imbd.expert_route(**ok)
    for bad in (dict(ws=None), dict(ws=ok["ws"][:-1]), dict(ws=ok["ws"].cpu()), dict(logits=z.double()), dict(gates=f(1000, 9)),
                dict(experts=ok["experts"].long()), dict(offsets=i(8)), dict(rows=i(1999)), dict(slots=i(2, 1000).t())):
        with pytest.raises((ValueError, TypeError, imbd.ImbdError)):
            imbd.expert_route(**{**ok, **bad})
    with pytest.raises(ValueError):
        imbd.expert_combine(y, i(4, 2), torch.empty(3, 64, device=dev))
    with pytest.raises(ValueError):
        imbd.expert_combine_bwd(y[:4], y, i(4, 2), f(4, 2), y[:, :-1])
    torch.cuda.synchronize()
    assert (y == 7.0).all() and (dw == 7.0).all() and (db == 7.0).all()


def test_two_streams_at_once(imbd, dev):
    """Calls on two streams share nothing: both give the bits that they give alone."""
    import torch
    Ls = [Layer(dev, [700, 0, 900], 512, 256, "bf16", gather=True, seed=s) for s in (1, 2)]
    alone = []
    for L in Ls:
        y = torch.zeros(L.n, 512, dtype=torch.bfloat16, device=dev)
        imbd.expert_fwd(L.w, L.x, L.offsets, y, bias=L.bias, rows=L.rows)
        alone.append(y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in Ls]
    outs = [torch.zeros_like(y) for y in alone]
    torch.cuda.synchronize()
    for _ in range(10):
        for L, s, y in zip(Ls, streams, outs):
            with torch.cuda.stream(s):
                imbd.expert_fwd(L.w, L.x, L.offsets, y, bias=L.bias, rows=L.rows)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))
