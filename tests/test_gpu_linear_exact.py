"""linear_fwd and linear_bwd on small whole numbers, bit for bit, over every kernel that takes a product.

All sums stay under 2^24 here, so fp32 holds them exactly in whatever order they are added, and what is stored has to be
equal: a range of K that is left out, counted twice or read from another call's workspace shows at every K, as does a column or
row next to what a tile covers. Stored as bf16 they are rounded once, to nearest, like a cast. What lies around the outputs and
behind the workspace has to stay as it is.

The smooth activations run over the large tiles' epilogues with the bounds of tests/test_gpu_linear.py."""
import pytest

from tests.test_gpu_expert import _dt, _gen, _padded
from tests.test_gpu_linear import ACTS, Layer, _check_bwd, _check_fwd
from tests.test_linear_launches import CASES, WIDE

pytestmark = pytest.mark.gpu

GUARD = 4096


class Whole(Layer):
    def __init__(self, dev, B, d_out, d_in, dtype, pad=0, seed=0):
        g = _gen(seed, dev)
        self.dev, self.B, self.d_out, self.d_in, self.dtype, self.dt, self.pad, self.g = dev, B, d_out, d_in, dtype, _dt(dtype), pad, g
        self.w, self.x = self.ints((d_out, d_in), 1), self.ints((B, d_in), 2)
        self.dy, self.z = self.ints((B, d_out), 2), self.ints((B, d_in), 2)
        self.bias = self.ints((1, d_out), 8, "f32", 0)[0]

    def ints(self, shape, most, dtype=None, pad=None):
        import torch
        dt, pad = _dt(dtype) if dtype else self.dt, self.pad if pad is None else pad
        v, _ = _padded(shape, shape[-1] + pad, dt, self.dev)
        v.copy_(torch.randint(-most, most + 1, shape, generator=self.g, device=self.dev, dtype=torch.int8))
        return v

    def room(self, B, d, dtype):
        """(an output, all of its memory): three rows more than it has, and columns between them."""
        import torch
        whole = torch.full((B + 3, d + self.pad), 7.0, dtype=_dt(dtype), device=self.dev)
        return whole[:B, :d], whole

    def workspace(self, imbd, which):
        import torch
        n = imbd.linear_workspace_bytes(which, imbd.dtype_code(self.dt), self.d_out, self.d_in, self.B)
        whole = torch.full((n + GUARD,), 255, dtype=torch.uint8, device=self.dev)
        return whole[:n] if n else None, whole[n:]


def _product(a, b):
    """a @ b of whole numbers; the products are exact in fp32 as well."""
    return (a.float() @ b.float()) if a.shape[0] * a.shape[1] + b.shape[0] * b.shape[1] > 1 << 28 else (a.double() @ b.double())


def _same(got, whole, ref, what):
    import torch
    ref = ref.float().to(got.dtype)
    bad = got != ref
    assert not bad.any(), (what, int(bad.sum()), bad.numel(), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), ref[bad][:4].tolist())
    around = whole.clone()
    around[:got.shape[0], :got.shape[1]] = 7.0
    assert torch.equal(around, torch.full_like(around, 7.0)), f"{what}: written around"


def _counted(imbd, tag, call):
    import torch
    imbd.timing_begin(imbd.IMBD_K_LINEAR, tag, 16)
    call()
    torch.cuda.synchronize()
    return imbd.timing_end()[0]


REDUCE, PAD = 3, 5  # layer tags of the sums' and the copies' launches


def _forward(imbd, L, act, out, residual, keep, ranged, copies, product):
    y, y_all = L.room(L.B, L.d_out, out)
    z, z_all = L.room(L.B, L.d_out, L.dtype)
    res, r = None, 0.0
    if residual:
        res = L.ints((L.B, L.d_out), 8, out)
        r = res.double()
        if residual == "in place":
            y.copy_(res)
            res = y
    for tag, n in ((REDUCE, int(ranged)), (PAD, copies)):
        if residual == "in place":
            y.copy_(r)
        ws, behind = L.workspace(imbd, 0)
        assert _counted(imbd, tag, lambda: imbd.linear_fwd(L.w, L.x, y, bias=L.bias, act=act, residual=res, z=z if keep else None, ws=ws)) == n
        assert (behind == 255).all()
    v = product + L.bias.double()
    if keep:
        _same(z, z_all, v, "z")
    else:
        assert (z_all == 7.0).all()
    _same(y, y_all, (v.clamp(min=0) if act == "relu" else v) + r, "y")


def _backward(imbd, L, which, act, out, residual, ranged, copies, dx_product, dw, db):
    dx, dx_all = L.room(L.B, L.d_in, out)
    gw, gw_all = L.room(L.d_out, L.d_in, "f32")
    gb, gb_all = L.room(1, L.d_out, "f32")
    res, r = None, 0.0
    if residual and "dx" in which:
        res = L.ints((L.B, L.d_in), 8, out)
        r = res.double()
        if residual == "in place":
            res = dx
    for tag, n in ((REDUCE, ranged), (PAD, copies)):
        if residual == "in place" and "dx" in which:
            dx.copy_(r)
        ws, behind = L.workspace(imbd, 1)
        got = _counted(imbd, tag, lambda: imbd.linear_bwd(
            L.w, L.dy, L.x, dw=gw if "dw" in which else None, db=gb[0] if "db" in which else None, dx=dx if "dx" in which else None,
            act=act, z=L.z if act != "none" else None, residual=res, ws=ws))
        assert (got > 0) == n if tag == REDUCE else got == n
        assert (behind == 255).all()
    for name, o, whole, ref in (("dw", gw, gw_all, dw), ("db", gb, gb_all, db)):
        if name in which:
            _same(o, whole, ref, name)
        else:
            assert (whole == 7.0).all()
    if "dx" in which:
        _same(dx, dx_all, (dx_product * (L.z.double() > 0) if act == "relu" else dx_product) + r, "dx")
    else:
        assert (dx_all == 7.0).all()


@pytest.mark.parametrize("pad", [0, 8])
@pytest.mark.parametrize("which,dtype,B,d_out,d_in,kernel,ranged,copies", CASES)
def test_whole_numbers(imbd, dev, which, dtype, B, d_out, d_in, kernel, ranged, copies, pad):
    L = Whole(dev, B, d_out, d_in, dtype, pad, seed=B + d_out)
    if which == "fwd":
        product = _product(L.x, L.w.t()).double()
        for act, out, residual, keep in (("none", "f32", None, False), ("relu", "bf16", "apart", True), ("none", "bf16", "in place", False),
                                         ("relu", "f32", "in place", True)):
            _forward(imbd, L, act, out, residual, keep, ranged, copies, product)
        return
    dx = _product(L.dy, L.w).double() if "dx" in which else None
    dw, db = _product(L.dy.t(), L.x), L.dy.double().sum(0)[None]
    for act, out, residual in (("none", "f32", None), ("relu", "bf16", "apart"), ("none", "bf16", "in place"), ("relu", "f32", "in place")):
        _backward(imbd, L, which, act, out, residual, ranged, copies, dx, dw, db)


@pytest.mark.parametrize("pad", [0, 8])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("which,dtype,B,d_out,d_in,kernel,ranged,copies",
                         [c for c in CASES if c[5] == WIDE and c[0] in ("fwd", "dx") and c[2] * c[3] * c[4] < 3 * 10 ** 10 and c[4] < 5000])
def test_activations_on_the_large_tiles(imbd, dev, which, dtype, B, d_out, d_in, kernel, ranged, copies, act, pad):
    L = Layer(dev, B, d_out, d_in, dtype, pad, seed=B)
    for residual, keep, out, in_place in ((True, True, "bf16", False), (True, False, "f32", True), (True, True, "bf16", True),
                                          (False, True, "f32", False), (False, False, "bf16", False)):
        if which == "fwd":
            _check_fwd(imbd, L, act, keep, residual, keep, out, in_place)
        else:
            _check_bwd(imbd, L, act, residual, out, "dx", in_place)


def test_gradients_of_no_rows_on_the_large_tiles(imbd, dev):
    """Without rows the gradients are zeros, whichever kernel writes them."""
    import torch
    for d_out, d_in, dtype in ((4104, 4096, "bf16"), (4099, 2500, "bf16"), (2049, 2050, "f32")):
        L = Whole(dev, 0, d_out, d_in, dtype)
        for which in ("dw db", "dw", "db"):
            gw, gw_all = L.room(d_out, d_in, "f32")
            gb, gb_all = L.room(1, d_out, "f32")
            imbd.linear_bwd(L.w, L.dy, L.x, dw=gw if "dw" in which else None, db=gb[0] if "db" in which else None,
                            dx=torch.empty(0, d_in, dtype=L.dt, device=dev), ws=L.workspace(imbd, 1)[0])
            for name, o, whole in (("dw", gw, gw_all), ("db", gb, gb_all)):
                if name in which:
                    _same(o, whole, torch.zeros_like(o), name)
                else:
                    assert (whole == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,d_out,d_in", [(4, 256, 512), (60, 256, 512), (400, 512, 256), (40, 67, 61), (2600, 2568, 2056)])
def test_infinities_reach_their_outputs(imbd, dev, B, d_out, d_in, dtype):
    """An infinite input makes a row's outputs infinite, NaN or zero as the formula does, and the other rows' stay finite."""
    import torch
    from tests.test_gpu_linear import _value, _ws
    for act in ACTS:
        L = Layer(dev, B, d_out, d_in, dtype)
        L.x[3, 0] = float("inf")
        y = torch.full((B, d_out), 7.0, dtype=L.dt, device=dev)
        imbd.linear_fwd(L.w, L.x, y, act=act, ws=_ws(imbd, 0, dtype, d_out, d_in, B, dev))
        ref = _value(act, L.x[3:4].double() @ L.w.double().t())[0]
        assert not ref.isfinite().all()
        got = y[3].double()
        assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.isinf(), ref.isinf())
        assert torch.equal(got[ref.isinf()], ref[ref.isinf()]) and (got[ref.isfinite()] == 0).all()
        assert y[:3].isfinite().all() and y[4:].isfinite().all()
