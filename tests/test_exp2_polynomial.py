"""The polynomial that stands for 2^x on the FMA units, read from the kernel's source: its error is what the comment beside it says."""
import os
import re

import numpy as np

SOURCE = os.path.join(os.path.dirname(__file__), "..", "paper_2602_11937_b200", "csrc", "prompt_attn.cu")


def test_relative_error():
    with open(SOURCE) as f:
        text = f.read()
    c = [np.float64(np.float32(re.search(r"kPoly%d = ([0-9.]+)f" % i, text).group(1))) for i in (5, 4, 3, 2, 1)] + [1.0]
    f = np.linspace(-0.5, 0.5, 1 << 20)
    p = np.full_like(f, c[0])
    for x in c[1:]:
        p = p * f + x
    exact = np.abs(p / np.exp2(f) - 1).max()
    assert 1.10e-7 < exact < 1.115e-7
    f32 = f.astype(np.float32)
    p = np.full_like(f32, c[0])
    for x in c[1:]:          # a product of two float32 is exact in float64; the sum's own rounding there is far below float32's
        p = (p.astype(np.float64) * f32.astype(np.float64) + x).astype(np.float32)
    assert np.abs(p.astype(np.float64) / np.exp2(f32.astype(np.float64)) - 1).max() < 1.56e-7
    assert "1.11e-7 at most, 1.55e-7 with float32's roundings" in text
