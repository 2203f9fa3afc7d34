"""Refusals of the expert layer's and AdamW's entry points, on the host: no device is touched."""
import ctypes

import numpy as np
import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_1712_04432_amd as m
    return m.load()


P = ctypes.c_void_p(256)
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, -1, -2, -4


def _route(lib, T=1000, E=8, k=2, renorm=1, logits=P, ldl=8, gates=P, experts=P, offsets=P, rows=P, slots=P, ws=P,
           ws_bytes=1 << 20):
    return lib.expert_route(T, E, k, renorm, logits, ldl, gates, experts, offsets, rows, slots, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,code", [
    (dict(T=-1), EINVAL), (dict(E=0), EINVAL), (dict(k=0), EINVAL), (dict(k=9), EINVAL),
    (dict(E=513, ldl=513), EUNSUPPORTED), (dict(E=32, ldl=32, k=17), EUNSUPPORTED), (dict(T=2 ** 30, k=2), EUNSUPPORTED),
    (dict(logits=None), EINVAL), (dict(gates=None), EINVAL), (dict(experts=None), EINVAL), (dict(offsets=None), EINVAL),
    (dict(rows=None), EINVAL), (dict(slots=None), EINVAL), (dict(ldl=7), EINVAL),
    (dict(ws=None), EWORKSPACE), (dict(ws_bytes=8), EWORKSPACE), (dict(ws=ctypes.c_void_p(264)), EINVAL)])
def test_route_refuses(lib, bad, code):
    assert _route(lib, **bad) == code
    assert lib.imbd_last_error()


def test_route_workspace(lib):
    assert lib.expert_route_workspace_bytes(-1, 8, 2) == 0
    assert lib.expert_route_workspace_bytes(16, 513, 2) == 0
    sizes = [lib.expert_route_workspace_bytes(T, 64, 8) for T in (1, 1000, 16384, 1 << 20, 1 << 26)]
    assert sizes[0] == 0 and sizes[1] > 0 and max(sizes) <= 256 * 64 * 4


@pytest.mark.parametrize("bad,code", [
    (dict(T=-1), EINVAL), (dict(k=9), EINVAL), (dict(E=600, lddl=600, ldl=600), EUNSUPPORTED), (dict(logits=None), EINVAL),
    (dict(logits=None, renorm=1), None), (dict(gates=None), EINVAL), (dict(experts=None), EINVAL),
    (dict(dgates=None), EINVAL), (dict(dlogits=None), EINVAL), (dict(ldl=7), EINVAL), (dict(lddl=7), EINVAL)])
def test_route_bwd_refuses(lib, bad, code):
    a = dict(T=100, E=8, k=2, renorm=0, logits=P, ldl=8, gates=P, experts=P, dgates=P, dlogits=P, lddl=8)
    a.update(bad)
    if code is None:
        a["T"] = 0  # (allowed: nothing to do)
        code = OK
    assert lib.expert_route_bwd(*a.values(), None) == code


FWD = dict(dtype=1, relu=0, E=4, d_out=64, d_in=32, n_rows=10, n_x=5, w=P, ldw=32, sw=2048, bias=None, x=P, ldx=32, rows=P,
           offsets=P, y=P, ldy=64, y_dtype=1)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), EINVAL), (dict(y_dtype=-1), EINVAL), (dict(E=0), EINVAL), (dict(E=513), EUNSUPPORTED),
    (dict(d_out=0), EINVAL), (dict(d_in=-3), EINVAL), (dict(n_rows=-1), EINVAL), (dict(n_x=-1), EINVAL),
    (dict(w=None), EINVAL), (dict(x=None), EINVAL), (dict(offsets=None), EINVAL), (dict(y=None), EINVAL),
    (dict(ldw=31), EINVAL), (dict(sw=2047), EINVAL), (dict(ldx=31), EINVAL), (dict(ldy=63), EINVAL),
    (dict(rows=None), EINVAL), (dict(n_rows=0, y=None, x=None, n_x=0), OK),
    (dict(n_rows=2 ** 31 - 1, n_x=2 ** 31 - 1, rows=None, d_out=2 ** 30, ldy=2 ** 30, sw=2 ** 40), EUNSUPPORTED)])
def test_fwd_refuses(lib, bad, code):
    assert lib.expert_fwd(*{**FWD, **bad}.values(), None) == code


BWD = dict(dtype=1, E=4, d_out=64, d_in=32, n_rows=10, n_x=5, w=P, ldw=32, sw=2048, dy=P, lddy=64, x=P, ldx=32, rows=P,
           offsets=P, dw=P, lddw=32, sdw=2048, db=P, dx=P, lddx=32, dx_dtype=1, mask_relu=1)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), EINVAL), (dict(dx_dtype=7), EINVAL), (dict(E=513), EUNSUPPORTED), (dict(d_out=0), EINVAL),
    (dict(dw=None, db=None, dx=None), EINVAL), (dict(offsets=None), EINVAL), (dict(dy=None), EINVAL),
    (dict(x=None), EINVAL), (dict(x=None, dw=None), EINVAL), (dict(w=None), EINVAL), (dict(ldw=31), EINVAL),
    (dict(sw=5), EINVAL), (dict(lddy=63), EINVAL), (dict(ldx=31), EINVAL), (dict(lddw=31), EINVAL), (dict(sdw=2047), EINVAL),
    (dict(lddx=31), EINVAL), (dict(rows=None), EINVAL)])
def test_bwd_refuses(lib, bad, code):
    assert lib.expert_bwd(*{**BWD, **bad}.values(), None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), EINVAL), (dict(y_dtype=2), EINVAL), (dict(T=-1), EINVAL), (dict(k=0), EINVAL),
    (dict(k=17), EUNSUPPORTED), (dict(d=0), EINVAL), (dict(n_rows=-1), EINVAL), (dict(ys=None), EINVAL),
    (dict(slots=None), EINVAL), (dict(y=None), EINVAL), (dict(ldys=31), EINVAL), (dict(ldy=31), EINVAL), (dict(T=0), OK)])
def test_combine_refuses(lib, bad, code):
    a = dict(dtype=1, T=10, k=2, d=32, n_rows=20, ys=P, ldys=32, slots=P, gates=None, y=P, ldy=32, y_dtype=1)
    a.update(bad)
    assert lib.expert_combine(*a.values(), None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), EINVAL), (dict(T=-1), EINVAL), (dict(k=17), EUNSUPPORTED), (dict(d=0), EINVAL), (dict(dy=None), EINVAL),
    (dict(slots=None), EINVAL), (dict(gates=None), EINVAL), (dict(dys=None), EINVAL), (dict(ys=None), EINVAL),
    (dict(lddy=31), EINVAL), (dict(ldys=31), EINVAL), (dict(lddys=31), EINVAL), (dict(T=0), OK)])
def test_combine_bwd_refuses(lib, bad, code):
    a = dict(dtype=1, T=10, k=2, d=32, n_rows=20, dy=P, lddy=32, ys=P, ldys=32, slots=P, gates=P, dys=P, lddys=32, dgates=P)
    a.update(bad)
    assert lib.expert_combine_bwd(*a.values(), None) == code


def _tensor(**kw):
    from paper_1712_04432_amd import AdamWTensor
    a = dict(w=4096, w_lp=None, grad=8192, m=12288, v=16384, m_scale=None, v_scale=None, n=1000, decay=0.0, grad_dtype=0,
             state_bits=32)
    a.update(kw)
    return AdamWTensor(*a.values())


def _array(*ts):
    from paper_1712_04432_amd import AdamWTensor
    return (AdamWTensor * len(ts))(*ts)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(grad_dtype=3), dict(state_bits=16), dict(decay=-0.5),
                                 dict(decay=float("nan")), dict(decay=float("inf")), dict(w=None), dict(grad=None),
                                 dict(m=None), dict(v=None), dict(state_bits=8), dict(state_bits=8, m_scale=64)])
def test_adamw_plan_refuses(lib, bad):
    arr = _array(_tensor(), _tensor(**bad))
    assert lib.adamw_plan_bytes(arr, 2) == 0
    assert lib.adamw_plan(arr, 2, P, 1 << 20) == EINVAL


@pytest.mark.parametrize("bad", [dict(w=4096), dict(w=4096 + 3996), dict(m=12288 + 4), dict(v=8192), dict(w_lp=16384 + 3998),
                                 dict(w=20480, m=20480 + 100, v=24576), dict(grad=4096),
                                 dict(state_bits=8, m=40000, v=41000, m_scale=42000, v_scale=42008)])
def test_adamw_plan_refuses_shared_memory(lib, bad):
    """Against a tensor of 1000 elements at 4096 (w), 8192 (gradient), 12288 and 16384 (states)."""
    apart = dict(w=1 << 20, grad=1 << 21, m=1 << 22, v=1 << 23)
    arr = _array(_tensor(**{**apart, **bad}), _tensor())
    assert lib.adamw_plan_bytes(arr, 2) == 0
    assert lib.adamw_plan(arr, 2, P, 1 << 20) == EINVAL and b"shares memory" in lib.imbd_last_error()
    for ok in (apart, {**apart, "grad": 8192}):  # (a gradient that two tensors read)
        assert lib.adamw_plan_bytes(_array(_tensor(**ok), _tensor()), 2) > 0


@pytest.mark.parametrize("bad", [dict(n_rows=2 ** 31 - 1, n_x=2 ** 31 - 1), dict(n_x=2 ** 31 - 1),
                                 dict(d_out=2 ** 30 + 8, ldy=2 ** 31, sw=2 ** 40), dict(d_in=2 ** 30 + 8, ldw=2 ** 31, ldx=2 ** 31, sw=2 ** 40)])
def test_fwd_refuses_sizes_past_32_bits(lib, bad):
    assert lib.expert_fwd(*{**FWD, **bad}.values(), None) == EUNSUPPORTED


def test_refuses_more_than_a_launch_takes(lib):
    """2^24 workgroups of 256 threads are 2^32 work-items."""
    tiles = dict(E=1, d_out=1, d_in=1, n_rows=2 ** 30, n_x=2 ** 30, rows=None, dtype=0, y_dtype=0, ldy=1, ldw=1, ldx=1)
    assert lib.expert_fwd(*{**FWD, **tiles}.values(), None) == EUNSUPPORTED
    T = 2 ** 29
    assert lib.expert_route_bwd(T, 8, 2, 1, None, 8, P, P, P, P, 8, None) == EUNSUPPORTED
    assert lib.expert_combine_bwd(0, T, 2, 8, 100, P, 8, P, 8, P, P, P, 8, P, None) == EUNSUPPORTED
    assert _route(lib, T=2 ** 31 - 1, k=1) == EUNSUPPORTED
    big = _array(_tensor(n=2 ** 37, w=1 << 42, grad=1 << 43, m=1 << 44, v=1 << 45))
    assert lib.adamw_plan_bytes(big, 1) == 0 and lib.adamw_plan(big, 1, P, 1 << 62) == EUNSUPPORTED


def test_adamw_plan(lib):
    """The plan covers every tensor once, whatever their sizes, and tensors of no elements cost nothing."""
    assert lib.adamw_plan_bytes(None, 0) == 0 and lib.adamw_plan(None, 0, None, 0) == OK
    assert lib.adamw_plan_bytes(None, 1) == 0 and lib.adamw_plan_bytes(_array(_tensor()), -1) == 0
    assert lib.adamw_plan_bytes(_array(_tensor(n=0, w=None)), 1) == 0
    one = lib.adamw_plan_bytes(_array(_tensor(n=1)), 1)
    big = dict(w=1 << 30, grad=1 << 31, m=1 << 32, v=1 << 33)
    arr = _array(_tensor(n=0), _tensor(n=100000, **big), _tensor(n=1))
    need = lib.adamw_plan_bytes(arr, 3)
    assert need > one > 0
    buf = np.zeros(need + 8, np.uint8)
    p = buf.ctypes.data
    assert lib.adamw_plan(arr, 3, p, need - 1) == EWORKSPACE
    assert lib.adamw_plan(arr, 3, None, need) == EINVAL
    assert lib.adamw_plan(arr, 3, p, need) == OK
    assert not buf[need:].any()


@pytest.mark.parametrize("bad", [dict(n=-1), dict(lr=float("nan")), dict(lr=float("inf")), dict(b1=1.0), dict(b1=-0.1),
                                 dict(b2=1.0), dict(b2=float("nan")), dict(eps=-1.0), dict(eps=float("inf")),
                                 dict(gs=float("nan")), dict(step=0), dict(plan=None), dict(plan=ctypes.c_void_p(8)),
                                 dict(size=7), dict(n=10 ** 6), dict(n=0)])
def test_adamw_step_refuses(lib, bad):
    size = lib.adamw_plan_bytes(_array(_tensor()), 1)
    a = dict(plan=P, size=size, n=1, lr=0.1, b1=0.9, b2=0.99, eps=1e-8, gs=1.0, step=1, dev=None)
    a.update(bad)
    assert lib.adamw_step(*a.values(), None) == EINVAL
    assert lib.adamw_step(None, 0, 0, 0.1, 0.9, 0.99, 1e-8, 1.0, 1, None, None) == OK


@pytest.mark.parametrize("dtype,d_in", [(0, 8), (1, 33)])
def test_bwd_launches_nothing_of_a_call_that_it_refuses(lib, dtype, d_in):
    """db has more tiles (2^24 of 64 rows) than a launch takes and dx has not: both are looked at before dx is launched,
    which without a device would be another error."""
    a = {**BWD, "dtype": dtype, "dx_dtype": dtype, "E": 1, "d_out": 2 ** 30, "d_in": d_in, "n_rows": 1, "n_x": 1,
         "rows": None, "ldw": d_in, "ldx": d_in, "lddx": d_in, "lddy": 2 ** 30, "mask_relu": 0, "dw": None}
    assert lib.expert_bwd(*a.values(), None) == EUNSUPPORTED and b"one launch" in lib.imbd_last_error()


class _Fake:
    """A tensor's description without memory: for calls that are refused before they reach the library."""

    def __init__(self, shape, dtype):
        import torch
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, "cuda:0"

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 256

    def numel(self):
        return self.shape.numel()

    def stride(self, i=None):
        s = [1]
        for d in reversed(self.shape[1:]):
            s.insert(0, s[0] * d)
        return tuple(s) if i is None else s[i]


@pytest.mark.parametrize("size", [2 ** 31, 2 ** 32])
def test_sizes_past_a_c_int_are_refused(lib, monkeypatch, size):
    """(As the low 32 bits of 2^32 they would be no rows at all: calls that do nothing and succeed.)"""
    import torch
    import types
    import paper_1712_04432_amd as m
    monkeypatch.setattr(m, "_here", lambda t, name: 0)
    monkeypatch.setattr(m, "_on", lambda stream, device: None)

    def b(*s):
        return _Fake(s, torch.bfloat16)

    def f(*s):
        return _Fake(s, torch.float32)

    def i(*s):
        return _Fake(s, torch.int32)

    B = size
    calls = [lambda: m.expert_route(f(B, 8), f(B, 2), i(B, 2), i(9), i(2 * B), i(B, 2)),
             lambda: m.expert_route(f(4, B), f(4, 2), i(4, 2), i(B + 1), i(8), i(4, 2)),
             lambda: m.expert_route_bwd(None, f(B, 2), i(B, 2), f(B, 2), f(B, 8)),
             lambda: m.expert_route_workspace_bytes(B, 8, 2),
             lambda: m.expert_fwd(b(2, 8, 8), b(B, 8), i(3), b(B, 8)),
             lambda: m.expert_fwd(b(2, 8, 8), b(B, 8), i(3), b(4, 8), rows=i(4)),
             lambda: m.expert_fwd(b(2, B, 8), b(4, 8), i(3), b(4, B)),
             lambda: m.expert_bwd(b(2, 8, 8), b(B, 8), b(B, 8), i(3), dx=b(B, 8)),
             lambda: m.expert_bwd(b(2, 8, B), b(4, 8), b(4, B), i(3), dw=f(2, 8, B)),
             lambda: m.expert_combine(b(4, 8), i(B, 2), b(B, 8)),
             lambda: m.expert_combine(b(B, 8), i(4, 2), b(4, 8)),
             lambda: m.expert_combine_bwd(b(B, 8), b(4, 8), i(B, 2), f(B, 2), b(4, 8), f(B, 2)),
             lambda: m.expert_combine_bwd(b(4, 8), b(B, 8), i(4, 2), f(4, 2), b(B, 8), f(4, 2)),
             lambda: m.adamw_step(types.SimpleNamespace(device=0), lr=0.1, step=size + 1)]
    for n, call in enumerate(calls):
        with pytest.raises(ValueError, match="under 2"):
            call()
            pytest.fail(f"call {n}")


@pytest.mark.parametrize("bad", [dict(eps=1e-46), dict(eps=1e-60), dict(lr=1e39), dict(lr=-1e300), dict(lr=1e38, b1=0.99)])
def test_adamw_step_refuses_what_fp32_does_not_hold(lib, bad):
    """An eps that fp32 makes zero (an element without gradients would be 0 / 0), a rate lr / (1 - beta1) that it makes
    infinite (0 * infinity)."""
    a = dict(plan=None, size=0, n=0, lr=0.1, b1=0.9, b2=0.99, eps=1e-8, gs=1.0, step=1, dev=None)
    for ok in ({}, dict(eps=0.0), dict(eps=1e-44), dict(lr=1e37, b1=0.0)):
        assert lib.adamw_step(*{**a, **ok}.values(), None) == OK
    assert lib.adamw_step(*{**a, **bad}.values(), None) == EINVAL and lib.imbd_last_error()


@pytest.mark.parametrize("bits,grad,lp", [(32, 0, 1), (32, 1, 0), (8, 1, 1), (8, 0, 0)])
def test_adamw_plan_goes_past_the_caches_by_the_sets_footprint(lib, bits, grad, lp):
    """Every array of the set counted once: up to 320 MiB through the caches, from 352 MiB on past them."""
    per = 4 + 2 * lp + (2 if grad else 4) + (2 if bits == 8 else 8)
    for mib, past in ((320, 0), (352, 8)):
        n = (mib << 20) // per // 2  # (two tensors)
        at = [dict(w=(1 << 44) + (i << 40), w_lp=(1 << 45) + (i << 40) if lp else None, grad=(1 << 46) + (i << 40),
                   m=(1 << 47) + (i << 40), v=(1 << 48) + (i << 40), m_scale=(1 << 49) + (i << 40),
                   v_scale=(1 << 50) + (i << 40)) for i in range(2)]
        arr = _array(*(_tensor(n=n, grad_dtype=grad, state_bits=bits, **a) for a in at))
        buf = np.zeros(lib.adamw_plan_bytes(arr, 2), np.uint8)
        assert lib.adamw_plan(arr, 2, buf.ctypes.data, len(buf)) == OK
        flags = buf[:144].view(np.int32).reshape(2, 18)[:, 17]  # the last word of each record
        assert (flags & 8 == past).all() and (flags & 3 == grad + (2 if bits == 8 else 0)).all()


@pytest.mark.parametrize("n", [2 ** 63 - 1, 2 ** 63 - 4000, 2 ** 62])
def test_adamw_plan_refuses_a_number_of_elements_past_64_bits(lib, n):
    arr = _array(_tensor(n=n))
    assert lib.adamw_plan_bytes(arr, 1) == 0 and lib.adamw_plan(arr, 1, P, 1 << 20) == EUNSUPPORTED
