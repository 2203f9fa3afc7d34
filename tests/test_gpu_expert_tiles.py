"""The products of any size on each of their tiles, at sizes that the rule of csrc/expert_tile.hip sends there.

Against 64 bits with the bounds of test_gpu_expert.py, whose own sizes all take tiles of 64 x 32."""
import pytest

from test_gpu_expert import Layer, _check_bwd, _check_fwd

pytestmark = pytest.mark.gpu

RAGGED = [0, 1, 1200, 64, 63, 129, 2000, 540]     # with the spare rows: 4000
LONG = [0, 20000, 1, 12997]
MANY = [(5 * e) % 17 for e in range(300)]


def tile(which, dtype, E, n, d_out, d_in):
    """The tile that the rule chooses (columns x rows)."""
    M = d_out if which == "fwd" else d_in

    def tiles(side):
        rows = E * -(-d_out // side) if which == "dw" else n // side + min(n, E) // 2
        return rows * -(-M // side)

    if dtype == "f32" and which != "dx":
        return "64x64" if tiles(64) >= 1024 else "64x32"
    return "128x64" if tiles(128) >= 256 else "64x32"


# (counts, d_out, d_in, the products that take the large tile): K of one product below one step (64 of bf16, 32 of
# fp32), of a whole number of steps and cut; columns that end inside a tile, inside 16 bytes, and fewer than 16 bytes
CASES = [(RAGGED, 1031, 1037, "fwd dx dw"), (RAGGED, 1031, 9, "fwd"), (RAGGED, 9, 1031, "dx"), (RAGGED, 1031, 128, "fwd"),
         (RAGGED, 128, 1031, "dx"), (RAGGED, 1031, 193, "fwd"), (LONG, 5, 67, "fwd dx"), (LONG, 67, 3, "fwd dx"),
         (MANY, 100, 5, "dw"), (MANY, 7, 133, "dw"), (MANY, 65, 1, "dw")]


def _layer(dev, counts, d_out, d_in, dtype, gather, pad, large):
    L = Layer(dev, counts, d_out, d_in, dtype, gather=gather, spare=3, pad=pad, seed=d_out + d_in)
    for which in large.split():
        got = tile(which, dtype, L.E, L.n, d_out, d_in)
        if dtype == "bf16" or which == "dx":
            assert got == "128x64", (which, got)
        else:
            assert got == "64x64" or d_out < 1000, (which, got)
    return L


@pytest.mark.parametrize("counts,d_out,d_in,large", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("pad", [0, 3])
def test_products_on_large_tiles(imbd, dev, counts, d_out, d_in, large, dtype, gather, pad):
    L = _layer(dev, counts, d_out, d_in, dtype, gather, pad, large)
    _check_fwd(imbd, L, relu=gather)
    _check_bwd(imbd, L, mask=not gather)


@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("f32", "bf16")])
def test_output_types_and_parts_on_large_tiles(imbd, dev, dtype, out):
    """The other output type, masks of gathered rows, and each output by itself with the bits that it has beside the
    others."""
    import torch
    L = _layer(dev, RAGGED, 1031, 1037, dtype, True, 5, "fwd dx dw")
    _check_fwd(imbd, L, bias=False, out=out)
    both = _check_bwd(imbd, L, mask=True, out=out)
    for i, which in enumerate(("dw", "db", "dx")):
        assert torch.equal(_check_bwd(imbd, L, mask=True, out=out, which=which)[i], both[i]), which
    db = torch.full_like(both[1], 7.0)
    imbd.expert_bwd(L.w, L.dy, None, L.offsets, db=db)
    assert torch.equal(db, both[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_outside_x_on_large_tiles(imbd, dev, dtype):
    import torch
    L = _layer(dev, RAGGED, 1031, 1037, dtype, True, 0, "fwd dx dw")
    bad = torch.tensor([-1, L.n_x, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=dev)
    L.rows[::7] = bad[torch.arange(len(L.rows[::7]), device=dev) % 4]
    _check_fwd(imbd, L)
    _check_bwd(imbd, L, mask=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nans_and_infinities_stay_in_their_rows_on_large_tiles(imbd, dev, dtype):
    """What is not finite in a slot behind an expert's last, or in one of its neighbours', reaches no sum of its own."""
    import torch
    clean, L = (_layer(dev, RAGGED, 1031, 1037, dtype, False, 0, "fwd dx dw") for _ in range(2))
    # slots 0 (expert 1) and 1264 (expert 3's last) among finite neighbours; the spare rows behind the last expert
    L.x[0], L.x[1264, 1036] = float("nan"), float("inf")
    L.x[L.used:], L.dy[L.used:] = float("nan"), float("inf")
    outs = []
    for l in (clean, L):
        y = torch.zeros(l.n, 1031, dtype=l.dt, device=dev)
        imbd.expert_fwd(l.w, l.x, l.offsets, y, bias=l.bias, relu=True)
        dw, db = torch.zeros(l.E, 1031, 1037, device=dev), torch.zeros(l.E, 1031, device=dev)
        dx = torch.zeros(l.n, 1037, dtype=l.dt, device=dev)
        imbd.expert_bwd(l.w, l.dy, l.x, l.offsets, dw=dw, db=db, dx=dx)
        outs.append((y, dw, db, dx))
    (yc, dwc, dbc, dxc), (y, dw, db, dx) = outs
    keep = torch.ones(L.n, dtype=torch.bool, device=dev)
    keep[[0, 1264]] = False
    assert torch.equal(y[keep], yc[keep]) and torch.isnan(y[0]).all()
    assert torch.equal(dx, dxc) and torch.equal(db, dbc)
    for e in (0, 2, 4, 5, 6, 7):
        assert torch.equal(dw[e], dwc[e]), e
    assert torch.isnan(dw[1]).all() and torch.equal(dw[3, :, :1036], dwc[3, :, :1036])
    assert not torch.isfinite(dw[3, :, 1036]).any()
