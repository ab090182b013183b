"""Packed tokens and caches whose offsets pass 32 bits, calls on several streams at once, and shapes drawn at random."""
import random

import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import BLOCK, D, KINDS, WEIGHT, attention64, cached, check, gen, make_starts
from test_gpu_chunk_attn import Case

pytestmark = pytest.mark.gpu


def test_rows_beyond_2_31_elements():
    """The last rows of arrays of more than 2^31 elements; all rows before belong to no sequence."""
    total, hkv, hq = 4_300_000, 1, 8
    new = [100, 33, 67]
    starts_list, starts = make_starts(new, total - 200)
    g = gen(3)
    q = torch.zeros(total, hq, D, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros(total, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    assert q.numel() > 2 ** 31
    for x in (q, k, v):
        x[-200:] = torch.randn(200, x.shape[1], D, generator=g, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    lse = torch.zeros(total, hq, device="cuda")
    desc = P.layer_desc(num_q_heads=hq, num_kv_heads=hkv)
    P.puzzle_prompt_attn(desc, q, k, v, starts, None, out, lse)
    torch.cuda.synchronize()
    for b in range(3):
        rows = slice(starts_list[b], starts_list[b + 1])
        want, want_lse, size = attention64(q[rows], k[rows].double(), v[rows].double(), 0, 0, None, desc.sm_scale)
        check("sequence %d" % b, out[rows], lse[rows], want, want_lse, size, WEIGHT["packed"])
    assert out[-300:-200].abs().max() == 0
    # the append's outputs and inputs at the same offsets
    blocks = 8
    caches = [torch.zeros(3 * blocks, hkv, BLOCK, D, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    lens = torch.tensor(new, dtype=torch.int32, device="cuda")
    view = P.kv_view(*caches, lens, max_blocks_per_seq=blocks)
    table = P.rope_table(128).cuda()
    out.zero_()
    P.puzzle_kv_append_packed(P.layer_desc(kv_dtype=P.KV_BF16, num_q_heads=hq, num_kv_heads=hkv), view, P.rope_view(table), q, k, v,
                              starts, out)
    torch.cuda.synchronize()
    x = q[starts_list[2]:starts_list[3]].float()
    c, s = table[:67, None, :32], table[:67, None, 32:]
    turned = torch.cat([x[..., :32] * c - x[..., 32:] * s, x[..., 32:] * c + x[..., :32] * s], -1).bfloat16()
    assert torch.equal(out[starts_list[2]:starts_list[3]], turned)
    assert torch.equal(caches[1][2 * blocks:].transpose(1, 2).flatten(0, 1)[:67], v[starts_list[2]:starts_list[3]])


@pytest.mark.parametrize("kv,num_blocks", [("bf16", 290_000), ("fp8", 560_000), ("fp4", 960_000)])
def test_caches_beyond_4_gib(kv, num_blocks):
    hkv, lens, new = 8, [300, 90], [20, 90]
    per_seq = 19
    shape, dtype = {"bf16": ((hkv, BLOCK, D), torch.bfloat16), "fp8": ((hkv, BLOCK, D), torch.uint8), "fp4": ((hkv, 576), torch.uint8)}[kv]
    c = Case(kv, lens, new, hkv=hkv)
    k, v = (torch.empty(num_blocks, *shape, dtype=dtype, device="cuda") for _ in "kv")
    assert k.nbytes > 1 << 32
    far = (num_blocks - 1 - torch.randperm(2 * per_seq, generator=gen(5), device="cuda")).int().view(2, per_seq)
    for x, small in ((k, c.k_cache), (v, c.v_cache)):
        x[far.flatten().long()] = small[c.blocks.flatten().long()]
    c.k_cache, c.v_cache, c.blocks, c.table = k, v, far, far
    c.call().verify()


def test_calls_on_two_streams_at_once():
    cases = [Case("fp8", [3000, 700], [40, 30], seed=1), Case("fp4", [2500, 900], [9, 300], seed=2)]
    want = []
    for c in cases:
        c.call().verify()
        want.append((c.out.clone(), c.lse.clone()))
        c.out.fill_(5)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(20):
        for c, s in zip(cases, streams):
            P.puzzle_chunk_attn(c.desc, c.view(), c.q, c.starts, c.sinks, c.out, c.lse, workspace=c.workspace, stream=s)
    torch.cuda.synchronize()
    for c, (out, lse) in zip(cases, want):
        assert torch.equal(c.out, out) and torch.equal(c.lse, lse)


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    r = random.Random(seed)
    kv = r.choice(list(KINDS))
    batch = r.choice((1, 2, 3, 7, 33))
    lens = [r.choice((r.randint(0, 40), r.randint(1, 700), r.randint(1, 3000))) for _ in range(batch)]
    new = [r.choice((0, 1, min(n, r.randint(1, 20)), r.randint(0, max(n, 1)))) for n in lens]
    c = Case(kv, lens, new, window=r.choice((0, 0, r.randint(1, 300))), hkv=r.choice((1, 2, 8)), seed=seed, table=r.random() < 0.7,
             first=r.choice((0, 5)), behind=r.choice((0, 70)), sinks=r.random() < 0.7)
    c.call().verify()
