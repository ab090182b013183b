"""Every pair's frequency of a stretched rotation table, with the ends of the ramp rounded to whole pairs and not."""
import math

import pytest
import torch


def _frequencies(table, rotary):
    """Angle of every pair at position 1 (at most 1, so it is the frequency) and the length of its row."""
    c, s = table.double()[1].view(2, rotary // 2)
    return torch.atan2(s, c), torch.hypot(s, c)


def _wanted(i, rotary, theta, factor, original, fast, slow, truncate):
    """One pair by the formula, with turns over the original context as the measure, written out pair by pair."""
    turns_of = lambda p: original * theta ** (-2.0 * p / rotary) / (2.0 * math.pi)
    ends = []
    for beta in (fast, slow):                                       # bisection: turns fall as the pair index grows
        a, b = -float(rotary), 4.0 * rotary
        for _ in range(200):
            m = (a + b) / 2.0
            a, b = (m, b) if turns_of(m) > beta else (a, m)
        ends.append((a + b) / 2.0)
    lo, hi = ends
    if truncate:
        lo, hi = math.floor(lo), math.ceil(hi)
    lo, hi = max(lo, 0), min(hi, rotary - 1)
    share = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)       # 0: unchanged, 1: divided
    f = theta ** (-2.0 * i / rotary)
    return f * (1.0 - share) + f / factor * share


@pytest.mark.parametrize("truncate", [True, False])
@pytest.mark.parametrize("rotary, theta, factor, original", [(64, 150000.0, 32.0, 4096), (64, 150000.0, 56.0, 4096),
                                                             (48, 10000.0, 4.0, 8192), (32, 500.0, 2.0, 2048)])
def test_every_pair_of_the_ramp(rotary, theta, factor, original, truncate):
    import paper_2602_11937_b200 as P
    table = P.rope_table(2, rotary, theta=theta, factor=factor, original_positions=original, truncate=truncate)
    got, gain = _frequencies(table, rotary)
    want = torch.tensor([_wanted(i, rotary, theta, factor, original, 32.0, 1.0, truncate) for i in range(rotary // 2)],
                        dtype=torch.float64)
    # two float32 entries of a size near the gain, half a step each: 2^-24 of the radius in the angle, times sqrt(2)
    assert torch.all((got - want).abs() <= 2.0 ** -23), (got / want - 1).abs().max()
    assert torch.all((gain - (0.1 * math.log(factor) + 1.0)).abs() <= 2.0 ** -22)


def test_the_two_conventions_differ_inside_the_ramp_only():
    import paper_2602_11937_b200 as P
    kw = dict(theta=150000.0, factor=32.0)
    a, b = (_frequencies(P.rope_table(2, 64, truncate=t, **kw), 64)[0] for t in (True, False))
    assert torch.equal(a[:9], b[:9]) and torch.equal(a[18:], b[18:])
    assert abs(float(a[13] / b[13]) - 1.054) < 1e-3                 # pair 13 of 32: 5.4 % apart
    c, d = (P.rope_table(9, 64, truncate=t, theta=150000.0) for t in (True, False))
    assert torch.equal(c, d)                                        # no stretching, no ramp


@pytest.mark.parametrize("bad", [dict(theta=1.0), dict(theta=0.0), dict(original_positions=0), dict(beta_fast=0.0),
                                 dict(beta_slow=-1.0), dict(beta_fast=1.0, beta_slow=2.0)])
def test_a_ramp_that_cannot_be_formed(bad):
    import paper_2602_11937_b200 as P
    with pytest.raises(ValueError):
        P.rope_table(4, 64, factor=2.0, **bad)
