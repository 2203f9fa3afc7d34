"""Refusals of the entry points of a layer with activation and residual, on the host: no device is touched."""
import ctypes

import pytest

from tests.test_expert_cpu import _Fake
from tests.test_vocab_cpu import _here

P, Q, R = ctypes.c_void_p(256), ctypes.c_void_p(1 << 40), ctypes.c_void_p(1 << 41)
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, -1, -2, -4


@pytest.fixture(scope="module")
def lib():
    import paper_1712_04432_amd as m
    return m.load()


FWD = dict(dtype=1, act=2, d_out=64, d_in=32, B=10, w=P, ldw=32, bias=P, x=P, ldx=32, residual=R, ldr=64, y=Q, ldy=64,
           y_dtype=1, z=ctypes.c_void_p(1 << 42), ldz=64, ws=P, ws_bytes=1 << 40)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), EINVAL), (dict(act=-1), EINVAL), (dict(act=5), EINVAL), (dict(d_out=0), EINVAL), (dict(d_in=0), EINVAL),
    (dict(B=-1), EINVAL), (dict(B=2 ** 31 - 1), EUNSUPPORTED), (dict(d_out=2 ** 30 + 1), EUNSUPPORTED), (dict(w=None), EINVAL),
    (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(y_dtype=3), EINVAL), (dict(ldw=31), EINVAL), (dict(ldx=31), EINVAL),
    (dict(ldy=63), EINVAL), (dict(ldr=63), EINVAL), (dict(ldz=63), EINVAL), (dict(residual=Q, ldr=65), EINVAL),
    (dict(z=Q), EINVAL), (dict(z=R), EINVAL), (dict(B=0, w=None, x=None, y=None), OK)])
def test_fwd_refuses(lib, bad, code):
    assert lib.linear_fwd(*{**FWD, **bad}.values(), None) == code
    assert code == OK or lib.imbd_last_error()


BWD = dict(dtype=1, act=2, d_out=64, d_in=32, B=10, w=P, ldw=32, dy=P, lddy=64, x=P, ldx=32, dw=Q, lddw=32, db=P, z=P, ldz=32,
           residual=R, ldr=32, dx=P, lddx=32, dx_dtype=1, ws=P, ws_bytes=1 << 40)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), EINVAL), (dict(act=9), EINVAL), (dict(d_out=0), EINVAL), (dict(d_in=-1), EINVAL), (dict(B=-1), EINVAL),
    (dict(dw=None, db=None, dx=None), EINVAL), (dict(dy=None), EINVAL), (dict(lddy=63), EINVAL), (dict(x=None), EINVAL),
    (dict(ldx=31), EINVAL), (dict(w=None), EINVAL), (dict(ldw=31), EINVAL), (dict(z=None), EINVAL), (dict(ldz=31), EINVAL),
    (dict(ldr=31), EINVAL), (dict(lddx=31), EINVAL), (dict(lddw=31), EINVAL), (dict(dx_dtype=4), EINVAL),
    (dict(residual=P, ldr=33), EINVAL)])
def test_bwd_refuses(lib, bad, code):
    assert lib.linear_bwd(*{**BWD, **bad}.values(), None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), EINVAL), (dict(act=5), EINVAL), (dict(B=-1), EINVAL), (dict(d=0), EINVAL), (dict(dy=None), EINVAL),
    (dict(z=None), EINVAL), (dict(dz=None), EINVAL), (dict(lddy=31), EINVAL), (dict(ldz=31), EINVAL), (dict(lddz=31), EINVAL),
    (dict(dz=P, lddz=40), EINVAL), (dict(B=0, dy=None), OK)])
def test_act_bwd_refuses(lib, bad, code):
    a = dict(dtype=1, act=2, B=10, d=32, dy=P, lddy=32, z=R, ldz=32, dz=Q, lddz=32)
    a.update(bad)
    assert lib.act_bwd(*a.values(), None) == code


SIZES = [(64, 32, 10), (4096, 4096, 8), (4096, 4096, 1), (16384, 4096, 64), (517, 1023, 1000), (1000, 4096, 300), (256, 784, 32768),
         (1, 1, 1), (8, 100000, 3), (4096, 4096, 200), (1024, 1024, 16384)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("d_out,d_in,B", SIZES)
def test_workspace(lib, d_out, d_in, B, dtype):
    """A call refuses less than it is told to bring, whatever the alignment of its tensors, and a workspace off its own."""
    size = dict(dtype=dtype, d_out=d_out, d_in=d_in, B=B)
    fwd = {**FWD, **size, "y_dtype": dtype, "ldw": d_in, "ldx": d_in, "ldr": d_out, "ldy": d_out, "ldz": d_out}
    bwd = {**BWD, **size, "dx_dtype": dtype, "ldw": d_in, "ldx": d_in, "lddw": d_in, "lddy": d_out, "ldz": d_in, "ldr": d_in,
           "lddx": d_in}
    for which, fn, a in ((0, lib.linear_fwd, fwd), (1, lib.linear_bwd, bwd)):
        need = lib.linear_workspace_bytes(which, dtype, d_out, d_in, B)
        if need:
            assert fn(*{**a, "ws_bytes": need - 1}.values(), None) == EWORKSPACE
            assert fn(*{**a, "ws": None}.values(), None) == EWORKSPACE
            assert fn(*{**a, "ws": ctypes.c_void_p(264)}.values(), None) == EINVAL
        assert need <= max(64 << 20, 16 * (d_out * d_in + B * max(d_in, d_out)))


def test_workspace_of_refused_sizes(lib):
    for bad in ((2, 1, 8, 8, 8), (-1, 1, 8, 8, 8), (0, 2, 8, 8, 8), (0, 1, 0, 8, 8), (1, 1, 8, 8, -1), (1, 0, 2 ** 30 + 1, 8, 8)):
        assert lib.linear_workspace_bytes(*bad) == 0


def test_refuses_more_than_a_launch_takes(lib):
    one = dict(dtype=0, d_out=1, d_in=1, B=2 ** 30, ldw=1, ldx=1, ldr=1, ldy=1, ldz=1, y_dtype=0)
    assert lib.linear_fwd(*{**FWD, **one}.values(), None) == EUNSUPPORTED and b"one launch" in lib.imbd_last_error()
    # dw's tiles are too many and dx's are not: both are looked at before dx is launched
    wide = {**BWD, "dtype": 0, "dx_dtype": 0, "d_out": 2 ** 30, "d_in": 1, "B": 1, "lddy": 2 ** 30, "ldw": 1, "ldx": 1, "lddw": 1,
            "ldz": 1, "ldr": 1, "lddx": 1}
    assert lib.linear_bwd(*wide.values(), None) == EUNSUPPORTED and b"one launch" in lib.imbd_last_error()


def test_tensors_that_do_not_fit_each_other_are_refused(lib, monkeypatch):
    import torch
    m = _here(monkeypatch)
    bf, f32 = torch.bfloat16, torch.float32

    def t(dt, *s):
        return _Fake(s, dt)

    good = dict(w=t(bf, 8, 4), x=t(bf, 3, 4), y=t(bf, 3, 8))
    for bad, err in ((dict(x=t(f32, 3, 4)), TypeError), (dict(x=t(bf, 3, 5)), ValueError), (dict(y=t(bf, 2, 8)), ValueError),
                     (dict(y=t(torch.float16, 3, 8)), TypeError), (dict(bias=t(bf, 8)), TypeError), (dict(bias=t(f32, 4)), ValueError),
                     (dict(residual=t(f32, 3, 8)), TypeError), (dict(residual=t(bf, 3, 4)), ValueError),
                     (dict(z=t(f32, 3, 8)), TypeError), (dict(act="tanh"), ValueError), (dict(act=None), ValueError)):
        with pytest.raises(err):
            m.linear_fwd(**{**good, **bad})
    good = dict(w=t(bf, 8, 4), dy=t(bf, 3, 8), x=t(bf, 3, 4), dw=t(f32, 8, 4), db=t(f32, 8), dx=t(bf, 3, 4))
    for bad, err in ((dict(dy=t(bf, 3, 4)), ValueError), (dict(x=t(bf, 2, 4)), ValueError), (dict(dw=t(bf, 8, 4)), TypeError),
                     (dict(db=t(f32, 4)), ValueError), (dict(dx=t(bf, 3, 8)), ValueError), (dict(z=t(f32, 3, 4)), TypeError),
                     (dict(residual=t(f32, 3, 4)), TypeError), (dict(act="elu"), ValueError)):
        with pytest.raises(err):
            m.linear_bwd(**{**good, **bad})
    for bad, err in ((dict(z=t(f32, 3, 8)), TypeError), (dict(dz=t(bf, 3, 4)), ValueError), (dict(act=""), ValueError)):
        with pytest.raises(err):
            m.act_bwd(**{**dict(dy=t(bf, 3, 8), z=t(bf, 3, 8), dz=t(bf, 3, 8), act="gelu"), **bad})


@pytest.mark.parametrize("size", [2 ** 31, 2 ** 32])
def test_sizes_past_a_c_int_are_refused(lib, monkeypatch, size):
    import torch
    m = _here(monkeypatch)

    def f(*s):
        return _Fake(s, torch.float32)

    B = size
    calls = [lambda: m.linear_fwd(f(8, 4), f(B, 4), f(B, 8)), lambda: m.linear_fwd(f(B, 4), f(3, 4), f(3, B)),
             lambda: m.linear_fwd(f(8, B), f(3, B), f(3, 8)), lambda: m.linear_bwd(f(8, 4), f(B, 8), f(B, 4), dx=f(B, 4)),
             lambda: m.linear_bwd(f(8, B), f(3, 8), f(3, B), dw=f(8, B)), lambda: m.act_bwd(f(B, 8), f(B, 8), f(B, 8), "relu"),
             lambda: m.linear_workspace_bytes(0, 1, 8, 8, B)]
    for n, call in enumerate(calls):
        with pytest.raises(ValueError, match="under 2"):
            call()
            pytest.fail(f"call {n}")
