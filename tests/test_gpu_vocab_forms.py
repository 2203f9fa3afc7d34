"""The forms of token_logprobs and distill_xent that a caller chooses by what it asks for: without entropy and lse, whose sums are
other kernels'; and that the timers see every launch. Tolerances as in tests/test_gpu_vocab.py."""
import pytest

from tests.test_gpu_expert import _gen
from tests.test_gpu_vocab import Exact, _logits, _near, _run_distill, _run_logprobs, _teacher, _tokens, _ws

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,V,launches", [(3, 40, 2), (300, 1000, 2), (2, 140000, 3)])
def test_distillation_is_timed_whole(imbd, dev, B, V, launches):
    """A row a workgroup and the batch's loss; long rows: parts' sums, parts, the loss."""
    z = _logits(dev, B, V, "f32")
    ids, t = _teacher(dev, B, V, 4)
    imbd.timing_begin(imbd.IMBD_K_DISTILL, -1, 16)
    _run_distill(imbd, z, ids, t, "f32")
    n, ms = imbd.timing_end()
    assert n == launches and ms > 0


def _run(imbd, z, tokens, n, temperature, entropy, lse):
    import torch
    B, V = z.shape
    dev = z.device
    logp, ent, ls = (torch.full((B,), 7.0, device=dev) for _ in range(3))
    ids = torch.full((B, n), 77, dtype=torch.int32, device=dev) if n else None
    top = torch.full((B, n), 7.0, device=dev) if n else None
    imbd.token_logprobs(z, tokens, logp, entropy=ent if entropy else None, lse=ls if lse else None, top_ids=ids, top_logp=top,
                        temperature=temperature, ws=_ws(imbd.token_logprobs_workspace_bytes(B, V, n), dev))
    torch.cuda.synchronize()
    assert entropy or (ent == 7.0).all()
    assert lse or (ls == 7.0).all()
    return logp, ent, ls, ids, top


KINDS = ["normal", "masked", "one_left", "lowest", "all_lowest", "ties", "constant", "ascending", "descending", "peaked", "large"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,V,kind", [(1, 1, "normal"), (3, 2, "normal")] +
                         [(*s, k) for s in ((5, 63), (3, 1000), (2, 9001), (2, 70001), (600, 2100), (1, 262147)) for k in KINDS])
def test_logprobs_without_entropy(imbd, dev, B, V, kind, dtype):
    """Log probabilities and alternatives as with it, rows in one workgroup and in parts; lse with and without."""
    import torch
    z, tokens = _logits(dev, B, V, dtype, kind, pad=3, seed=V), _tokens(dev, B, V)
    for n, t in ((0, 1.0), (0, 0.7), (20, 1.0), (64, 0.7)):
        x = Exact(z, t)
        zt = x.z.gather(1, tokens.clamp(0, V - 1).long()[:, None]).squeeze(1)
        ref = torch.where(tokens < 0, torch.zeros_like(zt), x.log_q(zt))
        ids = _run_logprobs(imbd, z, tokens, n, t)[3]
        for lse in (False, True):
            logp, _, ls, got, top = _run(imbd, z, tokens, n, t, False, lse)
            _near(logp, ref, x.tol_logq(zt), "logp")
            if lse:
                _near(ls, x.lse, x.tol_lse, "lse")
            if n:
                assert torch.equal(got, ids)
                zs = x.z.gather(1, ids.clamp(min=0).long())
                want = torch.where(ids >= 0, x.log_q(zs), torch.full_like(zs, -float("inf")))
                _near(top, want, x.tol_logq(zs), "top_logp")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [0, 4])
@pytest.mark.parametrize("V", [5, 3001, 100000])
def test_no_numbers_without_entropy(imbd, dev, V, n, dtype):
    """NaN, +inf and rows of -inf only make their own row NaN and nobody else's; a token past the end is NaN, no token 0."""
    import torch
    z = _logits(dev, 8, V, dtype)
    z[1, V // 2] = float("nan")
    z[2, V - 1] = float("inf")
    z[3] = -float("inf")
    z[7, 1] = -float("inf")
    tokens = torch.tensor([0, 1, 2, 3, V, 2 ** 31 - 1, -2 ** 31, 1], dtype=torch.int32, device=dev)
    logp, _, lse, ids, top = _run(imbd, z, tokens, n, 1.0, False, True)
    assert logp.isnan().tolist() == [False, True, True, True, True, True, False, False]
    assert logp[6] == 0 and logp[7] == -float("inf")
    assert lse.isnan().tolist() == [False, True, True, False, False, False, False, False] and lse[3] == -float("inf")
    if n:
        want = _run_logprobs(imbd, z, tokens, n)
        assert torch.equal(ids, want[3]) and ids[3].tolist() == [-1] * n and (top[3] == -float("inf")).all()
        assert top[1].isnan().all() and top[2].isnan().all() and not top[[0, 4, 5, 6, 7]].isnan().any()
