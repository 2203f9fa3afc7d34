"""The rational fit behind GELU (csrc/act.h) against the normal distribution's tail in 64 bits, on the host."""
import re
from pathlib import Path

import numpy as np

SOURCE = Path(__file__).resolve().parent.parent / "paper_1712_04432_amd" / "csrc" / "act.h"


def _coefficients():
    body = SOURCE.read_text().split("normal_tail(float u, float e) {")[1].split("return")[0]
    first = re.search(r"float p = (-?[\d.]+)f;", body).group(1)
    return [np.float32(c) for c in [first] + re.findall(r"p = fmaf\(p, t, (-?[\d.]+)f\);", body)]


def test_tail_of_the_normal_distribution():
    """e^(u^2 / 2) times the tail is erfcx(u / sqrt 2) / 2. As rounded the coefficients are good to 4.7e-8; evaluated in fp32
    (fused products, reciprocal to nearest) to 4e-7, of which every one of the ten steps may add a part of its half step."""
    from scipy.special import erfcx
    c = _coefficients()
    assert len(c) == 10
    u = np.concatenate([np.linspace(0, 64, 1 << 20), np.geomspace(64, 1e6, 1 << 16)]).astype(np.float32)
    ref = erfcx(u.astype(np.float64) / np.sqrt(2)) / 2
    t = 1 / (1 + u.astype(np.float64) / 4)
    p = np.zeros_like(t)
    for k in c:
        p = p * t + np.float64(k)
    assert np.abs(p * t / ref - 1).max() <= 4.7e-8
    t = (1 / (0.25 * u.astype(np.float64) + 1).astype(np.float32).astype(np.float64)).astype(np.float32)
    p = np.full_like(t, c[0])
    for k in c[1:]:  # (a product of two fp32 numbers is exact in 64 bits)
        p = (p.astype(np.float64) * t + np.float64(k)).astype(np.float32)
    assert np.abs((p * t).astype(np.float64) / ref - 1).max() <= 4e-7
