"""Logits of any size that float32 holds: rows whose logits are all far below or above zero, and references that rise from there.

Of a query only channels 0 and 1 are not zero.  A key's channel 0 is 0, 1 or 2 times the size or minus that, exact in every type, so that
large logits are either equal or far apart and their weights do not hang on the rounding of a float32; a key whose channel 0 is zero has a
logit of ordinary size by its channel 1.  Formula in 64 bits."""
import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import BLOCK, D, WEIGHT, attention64, check, gen, make_starts
from test_gpu_chunk_attn import Case

pytestmark = pytest.mark.gpu
SIZES = [159 / 128 * 2.0 ** e for e in (12, 19, 22, 24, 27, 30, 60, 110)]     # bf16 holds them; times a scale they take 32 bits
PATTERNS = ("low", "high", "late", "early", "rising")


def pattern(name, n):
    j = torch.arange(n, device="cuda")
    return {"low": -(1 + (j % 5 != 0).float()), "high": 1 + (j % 5 == 3).float(), "late": -(j < 2 * n // 3).float(),
            "early": -(j >= n // 3).float(), "rising": -(j % 64 < 40).float() * (1 + (j < n // 2).float())}[name]


def set_queries(q, size):
    q.zero_()
    q[:, :, 0] = size
    q[:, :, 1] = 8


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("window", [0, 70])
@pytest.mark.parametrize("name", PATTERNS)
def test_prompts(size, window, name):
    for hkv, new in ((2, [300, 70, 1]), (8, [1000])):
        hq, g = 8 * hkv, gen(5)
        at, starts = make_starts(new)
        q, k, v = (torch.randn(at[-1], h, D, generator=g, device="cuda").bfloat16() for h in (hq, hkv, hkv))
        set_queries(q, size)
        for b, n in enumerate(new):
            rows, x = slice(at[b], at[b + 1]), pattern(name, n)
            k[rows, :, 0] = x[:, None].bfloat16()
            k[rows, :, 1] *= (x == 0)[:, None]
        out, lse = torch.empty_like(q), torch.empty(at[-1], hq, device="cuda")
        P.puzzle_prompt_attn(P.layer_desc(window=window, num_q_heads=hq, num_kv_heads=hkv), q, k, v, starts, None, out, lse)
        for b in range(len(new)):
            rows = slice(at[b], at[b + 1])
            want, want_lse, bound = attention64(q[rows], k[rows].double(), v[rows].double(), 0, window, None, 0.125)
            check("%d" % b, out[rows], lse[rows], want, want_lse, bound, WEIGHT["packed"])


def set_keys(c, b, values):
    """Channels 0 and 1 of the keys of sequence b, unscaled; the 4-bit cache's block scales are 1."""
    n = len(values)
    j = torch.arange(n, device="cuda")
    blk, slot = c.blocks[b].long()[j // BLOCK], j % BLOCK
    pick = torch.randint(0, 8, (n,), generator=gen(b), device="cuda")
    second = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device="cuda")[pick] * (values == 0)
    if c.kv == "bf16":
        c.k_cache[blk, :, slot, 0] = values[:, None].bfloat16()
        c.k_cache[blk, :, slot, 1] = second[:, None].bfloat16() / 4
    elif c.kv == "fp8":
        c.k_cache[blk, :, slot, 0] = values.to(torch.float8_e4m3fn).view(torch.uint8)[:, None]
        c.k_cache[blk, :, slot, 1] = (second * 16).to(torch.float8_e4m3fn).view(torch.uint8)[:, None]
    else:
        c.k_cache[blk, :, 512:] = 0x38
        code = torch.tensor([0xC, 0xA, 0, 2, 4], device="cuda")[(values + 2).long()] | (pick * (values == 0)) << 4
        c.k_cache[blk, :, 32 * slot] = code.to(torch.uint8)[:, None]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("kv", ["fp8", "bf16", "fp4"])
@pytest.mark.parametrize("window", [0, 70])
@pytest.mark.parametrize("name", PATTERNS)
def test_chunks(kv, size, window, name):
    for hkv, lens, new in ((2, [500, 90, 17], [60, 90, 1]), (8, [1500], [700])):
        c = Case(kv, lens, new, window, hkv=hkv, sinks=False)
        set_queries(c.q, size)
        for b, n in enumerate(lens):
            set_keys(c, b, pattern(name, n))
        c.call().verify()


@pytest.mark.parametrize("kv", ["fp8", "bf16", "fp4"])
@pytest.mark.parametrize("name", ["late", "early"])
@pytest.mark.parametrize("sinks", [False, True])
def test_parts(kv, name, sinks):
    """The keys of a sequence cut into parts, some of which have nothing but the large logits."""
    c = Case(kv, [20000], [5], hkv=8, sinks=sinks)
    set_queries(c.q, SIZES[6])
    set_keys(c, 0, pattern(name, 20000))
    before = P.puzzle_launch_count()
    c.call().verify()
    assert P.puzzle_launch_count() - before == 2
