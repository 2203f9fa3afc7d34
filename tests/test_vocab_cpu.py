"""Refusals of the entry points for a vocabulary's logits, on the host: no device is touched."""
import ctypes

import pytest

from tests.test_expert_cpu import _Fake

P, Q = ctypes.c_void_p(256), ctypes.c_void_p(1 << 40)
OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, -1, -2, -4
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    import paper_1712_04432_amd as m
    return m.load()


DISTILL = dict(dtype=1, B=10, V=100, K=4, logits=P, ldz=100, ids=P, teacher=P, lse=None, weight=None, temperature=1.0,
               inv_batch=0.1, loss=P, row_loss=P, dlogits=Q, lddl=100, dlogits_dtype=1, ws=P, ws_bytes=1 << 30)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), EINVAL), (dict(B=-1), EINVAL), (dict(V=0), EINVAL), (dict(K=0), EINVAL), (dict(K=257), EUNSUPPORTED),
    (dict(B=1 << 24), EUNSUPPORTED), (dict(V=(1 << 30) + 1, ldz=1 << 31, lddl=1 << 31), EUNSUPPORTED),
    (dict(logits=None), EINVAL), (dict(ids=None), EINVAL), (dict(teacher=None), EINVAL), (dict(loss=None), EINVAL),
    (dict(row_loss=None), EINVAL), (dict(ldz=99), EINVAL), (dict(lddl=99), EINVAL), (dict(dlogits_dtype=5), EINVAL),
    (dict(dlogits=P, lddl=101), EINVAL), (dict(dlogits=P, dlogits_dtype=0), EINVAL),
    (dict(temperature=0.0), EINVAL), (dict(temperature=-1.0), EINVAL), (dict(temperature=NAN), EINVAL),
    (dict(temperature=INF), EINVAL), (dict(temperature=1e-39), EINVAL), (dict(temperature=1e20), EINVAL),
    (dict(inv_batch=INF), EINVAL), (dict(inv_batch=NAN), EINVAL)])
def test_distill_refuses(lib, bad, code):
    assert lib.distill_xent(*{**DISTILL, **bad}.values(), None) == code
    assert lib.imbd_last_error()


LOGPROBS = dict(dtype=1, B=10, V=100, n=4, logits=P, ldz=100, tokens=P, temperature=1.0, logp=P, entropy=P, lse=P, top_ids=P,
                top_logp=P, ws=P, ws_bytes=1 << 30)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), EINVAL), (dict(B=-1), EINVAL), (dict(V=0), EINVAL), (dict(n=-1), EINVAL), (dict(n=65), EUNSUPPORTED),
    (dict(B=1 << 24), EUNSUPPORTED), (dict(V=(1 << 30) + 1, ldz=1 << 31), EUNSUPPORTED), (dict(logits=None), EINVAL),
    (dict(tokens=None), EINVAL), (dict(logp=None), EINVAL), (dict(top_ids=None), EINVAL), (dict(top_logp=None), EINVAL),
    (dict(ldz=99), EINVAL), (dict(temperature=0.0), EINVAL), (dict(temperature=NAN), EINVAL), (dict(B=0, logits=None), OK)])
def test_logprobs_refuses(lib, bad, code):
    assert lib.token_logprobs(*{**LOGPROBS, **bad}.values(), None) == code


LOGPROBS_BWD = dict(dtype=1, B=10, V=100, logits=P, ldz=100, tokens=P, temperature=1.0, lse=P, entropy=P, dlogp=P, dentropy=P,
                    dlogits=Q, lddl=100, dlogits_dtype=1)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), EINVAL), (dict(B=-1), EINVAL), (dict(V=0), EINVAL), (dict(B=1 << 24), EUNSUPPORTED),
    (dict(logits=None), EINVAL), (dict(tokens=None), EINVAL), (dict(lse=None), EINVAL), (dict(entropy=None), EINVAL),
    (dict(dlogits=None), EINVAL), (dict(ldz=99), EINVAL), (dict(lddl=99), EINVAL), (dict(dlogits_dtype=-1), EINVAL),
    (dict(dlogits=P, lddl=104), EINVAL), (dict(dlogits=P, dlogits_dtype=0), EINVAL), (dict(temperature=INF), EINVAL),
    (dict(B=0, dlogits=None), OK)])
def test_logprobs_bwd_refuses(lib, bad, code):
    assert lib.token_logprobs_bwd(*{**LOGPROBS_BWD, **bad}.values(), None) == code


def test_workspaces(lib):
    """What a call is told to bring it accepts, and no less; sizes that it refuses need none."""
    for B, V, n in ((1, 131072, 20), (16, 131072, 64), (1, 1 << 30, 64), (4096, 131072, 5), (3, 7, 7)):
        need = lib.token_logprobs_workspace_bytes(B, V, n)
        if need:
            a = {**LOGPROBS, "B": B, "V": V, "n": n, "ldz": V}
            assert lib.token_logprobs(*{**a, "ws_bytes": need - 1}.values(), None) == EWORKSPACE
            assert lib.token_logprobs(*{**a, "ws": None}.values(), None) == EWORKSPACE
            assert lib.token_logprobs(*{**a, "ws": ctypes.c_void_p(264)}.values(), None) == EINVAL
        need = lib.distill_workspace_bytes(B, V, max(1, n))
        if need:
            a = {**DISTILL, "B": B, "V": V, "K": max(1, n), "ldz": V, "lddl": V}
            assert lib.distill_xent(*{**a, "ws_bytes": need - 1}.values(), None) == EWORKSPACE
    assert lib.token_logprobs_workspace_bytes(-1, 10, 1) == 0 and lib.token_logprobs_workspace_bytes(1, 10, 65) == 0
    assert lib.distill_workspace_bytes(1, 0, 1) == 0 and lib.distill_workspace_bytes(1, 10, 0) == 0


def _here(monkeypatch):
    import paper_1712_04432_amd as m
    monkeypatch.setattr(m, "_here", lambda t, name: 0)
    monkeypatch.setattr(m, "_on", lambda stream, device: None)
    return m


@pytest.mark.parametrize("size", [2 ** 31, 2 ** 32])
def test_sizes_past_a_c_int_are_refused(lib, monkeypatch, size):
    import torch
    m = _here(monkeypatch)
    f32, i32 = torch.float32, torch.int32

    def f(*s):
        return _Fake(s, f32)

    def i(*s):
        return _Fake(s, i32)

    B = size
    calls = [lambda: m.distill_xent(f(B, 8), i(B, 2), f(B, 2), 1.0, f(1), f(B)),
             lambda: m.distill_xent(f(4, B), i(4, 2), f(4, 2), 1.0, f(1), f(4)),
             lambda: m.distill_xent(f(4, 8), i(4, B), f(4, B), 1.0, f(1), f(4)),
             lambda: m.token_logprobs(f(B, 8), i(B), f(B)), lambda: m.token_logprobs(f(4, B), i(4), f(4)),
             lambda: m.token_logprobs(f(4, 8), i(4), f(4), top_ids=i(4, B), top_logp=f(4, B)),
             lambda: m.token_logprobs_bwd(f(B, 8), i(B), f(B), f(B, 8)),
             lambda: m.token_logprobs_bwd(f(4, B), i(4), f(4), f(4, B)),
             lambda: m.distill_workspace_bytes(B, 8, 2), lambda: m.token_logprobs_workspace_bytes(4, B, 2)]
    for n, call in enumerate(calls):
        with pytest.raises(ValueError, match="under 2"):
            call()
            pytest.fail(f"call {n}")


def test_tensors_that_do_not_fit_each_other_are_refused(lib, monkeypatch):
    import torch
    m = _here(monkeypatch)
    f32, i32, i64, f64 = torch.float32, torch.int32, torch.int64, torch.float64

    def t(dt, *s):
        return _Fake(s, dt)

    good = dict(logits=t(f32, 4, 8), ids=t(i32, 4, 2), teacher=t(f32, 4, 2), inv_batch=1.0, loss=t(f32, 1), row_loss=t(f32, 4))
    for bad, err in ((dict(ids=t(i64, 4, 2)), TypeError), (dict(ids=t(i32, 3, 2)), ValueError),
                     (dict(teacher=t(f32, 4, 3)), ValueError), (dict(teacher=t(f64, 4, 2)), TypeError),
                     (dict(loss=t(f32, 2)), ValueError), (dict(row_loss=t(f32, 5)), ValueError),
                     (dict(logits=t(torch.float16, 4, 8)), TypeError), (dict(dlogits=t(f32, 4, 9)), ValueError),
                     (dict(lse=t(f32, 3)), ValueError), (dict(weight=t(f64, 4)), TypeError)):
        with pytest.raises(err):
            m.distill_xent(**{**good, **bad})
    good = dict(logits=t(f32, 4, 8), tokens=t(i32, 4), logp=t(f32, 4))
    for bad, err in ((dict(tokens=t(i64, 4)), TypeError), (dict(tokens=t(i32, 5)), ValueError),
                     (dict(logp=t(f32, 4, 1)), ValueError), (dict(entropy=t(f32, 3)), ValueError),
                     (dict(top_ids=t(i32, 4, 2), top_logp=t(f32, 4, 3)), ValueError),
                     (dict(top_logp=t(f32, 4, 2)), ValueError), (dict(lse=t(f64, 4)), TypeError)):
        with pytest.raises(err):
            m.token_logprobs(**{**good, **bad})
    good = dict(logits=t(f32, 4, 8), tokens=t(i32, 4), lse=t(f32, 4), dlogits=t(f32, 4, 8))
    for bad, err in ((dict(dlogits=t(f32, 8, 4)), ValueError), (dict(dlogp=t(f32, 3)), ValueError),
                     (dict(dentropy=t(f64, 4)), TypeError), (dict(dlogits=t(torch.float16, 4, 8)), TypeError)):
        with pytest.raises(err):
            m.token_logprobs_bwd(**{**good, **bad})
