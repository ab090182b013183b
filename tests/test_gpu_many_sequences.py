"""Batches of up to 4096 sequences of packed tokens, most of them short or empty."""
import random

import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import D, FLOOR, WEIGHT, attention64, check, gen, make_starts
from test_gpu_append_packed import Case as Append, same_bytes
from test_gpu_chunk_attn import Case as Chunk

pytestmark = pytest.mark.gpu


def ragged(batch, most, seed):
    r = random.Random(seed)
    return [r.choice((0, 1, r.randint(0, most))) for _ in range(batch)]


@pytest.mark.parametrize("kv", ["fp8", "bf16", "fp4"])
@pytest.mark.parametrize("batch, most", [(300, 70), (4096, 5)])
def test_append(kv, batch, most):
    new = ragged(batch, most, batch)
    new[-1] = most
    c = Append(kv, [n + b % 40 for b, n in enumerate(new)], new, hkv=1)
    want = [x.clone() for x in c.caches]
    out = c.rectangle(want)
    c.call()
    assert c.status.item() == 0 and same_bytes(c.caches, want)
    for b in range(0, batch, 7):
        assert torch.equal(c.q_out[c.at[b]:c.at[b + 1]], out[b, :new[b]])


@pytest.mark.parametrize("batch, most, window", [(300, 90, 0), (4096, 6, 0), (1000, 40, 20)])
def test_prompts(batch, most, window):
    new = ragged(batch, most, batch + 1)
    new[-1] = most
    hkv, hq, g = 1, 8, gen(1)
    at, starts = make_starts(new)
    q, k, v = (torch.randn(at[-1], h, D, generator=g, device="cuda").bfloat16() for h in (hq, hkv, hkv))
    out, lse = torch.full_like(q, 7), torch.full((at[-1], hq), 7.0, device="cuda")
    P.puzzle_prompt_attn(P.layer_desc(window=window, num_q_heads=hq, num_kv_heads=hkv), q, k, v, starts, None, out, lse)
    assert not ((out == 7).all(-1) & (lse == 7)).any()
    for b in list(range(0, batch, batch // 40)) + [batch - 1]:
        if new[b]:
            rows = slice(at[b], at[b + 1])
            want, want_lse, size = attention64(q[rows], k[rows].double(), v[rows].double(), 0, window, None, 0.125)
            check("sequence %d" % b, out[rows], lse[rows], want, want_lse, size, WEIGHT["packed"])


@pytest.mark.parametrize("kv", ["fp8", "bf16", "fp4"])
@pytest.mark.parametrize("batch, most", [(300, 30), (4096, 3)])
def test_chunks(kv, batch, most):
    new = ragged(batch, most, batch + 2)
    new[-1] = most
    c = Chunk(kv, [n + b * 37 % 200 for b, n in enumerate(new)], new, hkv=1).call()
    assert c.status.item() == 0
    assert not ((c.out == 7).all(-1) & (c.lse == 7)).any()
    for b in list(range(0, batch, batch // 40)) + [batch - 1]:
        if new[b]:
            rows, m = slice(c.at[b], c.at[b + 1]), c.lens[b]
            want, lse, size = attention64(c.q[rows], c.keys(b, m, False), c.keys(b, m, True), m - new[b], 0, c.sinks, 0.125, FLOOR[kv])
            check("sequence %d" % b, c.out[rows], c.lse[rows], want, lse, size, WEIGHT[kv])
