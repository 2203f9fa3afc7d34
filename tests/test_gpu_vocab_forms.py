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
