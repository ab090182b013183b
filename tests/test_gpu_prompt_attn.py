"""Attention of whole packed prompts against the formula in 64 bits."""
import math

import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import D, WEIGHT, attention64, check, gen, make_starts

pytestmark = pytest.mark.gpu


def run(new, window=0, sinks=True, hkv=8, seed=1, first=0, behind=0, sliced=True, fix=None, sm_scale=None, mangle=None):
    """Prompts of `new` tokens from row `first` on, `behind` rows behind the last; returns what the kernel left and wrote."""
    hq = 8 * hkv
    g = gen(seed)
    at, starts = make_starts(new, first)
    total = at[-1] + behind
    if sliced:
        qkv = torch.randn(total, hq + 2 * hkv, D, generator=g, device="cuda").bfloat16()
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    else:
        q, k, v = (torch.randn(total, h, D, generator=g, device="cuda").bfloat16() for h in (hq, hkv, hkv))
    if mangle:
        mangle(q, k, v, at)
    sk = torch.randn(hq, generator=g, device="cuda") if sinks else None
    out = torch.full((total, hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((total, hq), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = P.layer_desc(window=window, num_q_heads=hq, num_kv_heads=hkv, sm_scale=sm_scale)
    P.puzzle_prompt_attn(desc, q, k, v, starts, sk, out, lse, dev_status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    if fix:
        fix(out, lse)
    scale = desc.sm_scale
    for b, n in enumerate(new):
        if n:
            rows = slice(at[b], at[b + 1])
            want, want_lse, size = attention64(q[rows], k[rows].double(), v[rows].double(), 0, window, sk, scale)
            check("prompt %d of %s" % (b, new), out[rows], lse[rows], want, want_lse, size, WEIGHT["packed"])
    assert (out[:first] == 7).all() and (lse[:first] == 7).all()
    assert (out[at[-1]:] == 7).all() and (lse[at[-1]:] == 7).all()
    return out, lse


@pytest.mark.parametrize("new", [[1], [2], [15], [16], [17], [32], [33], [127], [128], [129], [255], [257], [300, 1, 0, 41],
                                 [0, 0, 5], [640], [1000, 999]])
@pytest.mark.parametrize("window", [0, 1, 128])
def test_lengths(new, window):
    run(new, window)


@pytest.mark.parametrize("window", [2, 15, 16, 17, 100, 129, 500, 2 ** 31 - 1])
def test_windows(window):
    run([700, 33], window, seed=window % 1000)


def test_no_sinks():
    run([200, 7], sinks=False)
    run([200, 7], window=30, sinks=False)


@pytest.mark.parametrize("hkv", [1, 2, 5, 16])
def test_heads(hkv):
    run([130, 64, 3], hkv=hkv)


def test_contiguous_rows():
    run([77, 200], sliced=False)


def test_rows_of_no_sequence_stay():
    run([70, 0, 40], first=5, behind=9)


def test_many_sequences():
    run([(7 * i) % 40 for i in range(70)])


def test_wide_groups():
    """Enough tokens for groups of 32, whose second half can be missing or short."""
    run([500, 17, 1200, 16, 48, 801])
    run([500, 17, 1200, 16, 48, 801], window=128)


def test_large_logits():
    """Maxima that grow along the keys, so that the reference is raised again and again."""
    def mangle(q, k, v, at):
        k *= (1 + torch.arange(k.shape[0], device="cuda") / 60.0)[:, None, None]
    run([900], mangle=mangle)


@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_values_that_a_row_does_not_see(what):
    """An infinity or NaN in a value is in the sum of the rows that see it and of no other."""
    def mangle(q, k, v, at):
        for row, head, channel in ((40, 0, 3), (150, 0, 3), (150, 2, 60), (299, 1, 0)):
            v[row, head, channel] = what
    for window in (0, 20, 130):
        run([300, 100], window, mangle=mangle, hkv=3)


def test_keys_that_a_row_does_not_see():
    hq = 16
    got = {}
    for bad in (False, True):
        g = gen(3)
        q, k, v = (torch.randn(400, h, D, generator=g, device="cuda").bfloat16() for h in (hq, 2, 2))
        if bad:
            k[170, 0, 5] = math.nan
        o = torch.empty(400, hq, D, dtype=torch.bfloat16, device="cuda")
        starts = make_starts([300, 100])[1]
        P.puzzle_prompt_attn(P.layer_desc(num_q_heads=hq, num_kv_heads=2), q, k, v, starts, None, o)
        got[bad] = o
    assert torch.equal(got[True][:170], got[False][:170]) and torch.equal(got[True][300:], got[False][300:])
    assert torch.equal(got[True][:, 8:], got[False][:, 8:])
    assert got[True][170:300, :8].isnan().all()


@pytest.mark.parametrize("scale", [-0.125, 0.0, 1e-30, 3.0])
def test_scales(scale):
    run([200], sm_scale=scale, window=150)


def test_the_same_bits_twice():
    a, b = run([900, 333], seed=5), run([900, 333], seed=5)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
