"""imbd_timing_begin takes every kernel class of the header, on the host (tests/_launched.py: the events are refused, for want of
a device, once the request is accepted)."""
import re
from pathlib import Path

from tests._launched import ROOT, launched


def test_every_class_can_be_timed():
    import paper_1712_04432_amd._abi as abi
    text = re.search(r"enum imbd_kernel_class \{(.*?)\}", (Path(ROOT) / "include" / "imbd.h").read_text(), re.S).group(1)
    classes = {k: int(v) for k, v in re.findall(r"(IMBD_K_\w+) = (\d+)", text)}
    count = classes.pop("IMBD_K_COUNT")
    assert sorted(classes.values()) == list(range(count)) and abi.IMBD_K_COUNT == count
    assert all(getattr(abi, k) == v for k, v in classes.items())
    got = launched([("imbd_timing_begin", [c, -1, 4]) for c in range(count)])
    assert all(code == -3 and "hipEventCreate" in text for code, text in got), got
    assert [code for code, _ in launched([("imbd_timing_begin", a) for a in ([-1, -1, 4], [count, -1, 4], [0, -1, 0])])] == [-1] * 3
