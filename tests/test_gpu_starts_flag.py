"""A bad entry of starts is reported wherever in a large batch it stands."""
import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import D, gen
from test_gpu_chunk_attn import Case

pytestmark = pytest.mark.gpu


def bad(batch, at, total):
    s = torch.full((batch + 1,), total, dtype=torch.int32)
    s[0], s[at] = 0, 99
    return s.cuda()


@pytest.mark.parametrize("total", [1, 5])
@pytest.mark.parametrize("batch, at", [(3, 2), (32, 31), (40, 36), (1000, 70), (1000, 999), (4096, 4095)])
def test_reported(batch, at, total):
    g = gen(1)
    q, k, v = (torch.randn(total, h, D, generator=g, device="cuda").bfloat16() for h in (16, 2, 2))
    out = torch.full((total, 16, D), 7.0, dtype=torch.bfloat16, device="cuda")
    starts = bad(batch, at, total)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = P.layer_desc(num_q_heads=16, num_kv_heads=2)
    P.puzzle_prompt_attn(desc, q, k, v, starts, None, out, dev_status=status)
    assert status.item() == P.DEV_BAD_STARTS
    want = torch.empty_like(out)
    P.puzzle_prompt_attn(desc, q, k, v, torch.tensor([0, total], dtype=torch.int32, device="cuda"), None, want)
    assert torch.equal(out, want)
    for kv in ("fp8", "bf16", "fp4"):
        c = Case(kv, [20] * batch, [total] + [0] * (batch - 1), hkv=1, per_seq=2)
        c.call().verify()
        c.starts = starts
        c.call().verify(status=P.DEV_BAD_STARTS)


@pytest.mark.parametrize("batch, at", [(3, 2), (40, 36), (4096, 4095)])
def test_reported_by_the_append(batch, at):
    k, v = (torch.randn(5, 2, D, device="cuda").bfloat16() for _ in "kv")
    caches = [torch.zeros(batch, 2, 16, D, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    lens = torch.full((batch,), 5, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    desc = P.layer_desc(kv_dtype=P.KV_BF16, num_q_heads=16, num_kv_heads=2)
    P.puzzle_kv_append_packed(desc, P.kv_view(*caches, lens, max_blocks_per_seq=1), None, None, k, v, bad(batch, at, 5), dev_status=status)
    assert status.item() == P.DEV_BAD_STARTS
    assert torch.equal(caches[0][0].transpose(0, 1)[:5], k)
