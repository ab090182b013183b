"""Many calls on the same inputs, alone and beside another stream's, give the same bits: a product that ran before the one whose
operand it overwrites had ended would show here."""
import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import D, gen, make_starts
from test_gpu_chunk_attn import Case

pytestmark = pytest.mark.gpu


def repeats(call, buffers):
    call(None)
    torch.cuda.synchronize()
    want = [b.clone() for b in buffers]
    side, x = torch.cuda.Stream(), torch.randn(2048, 2048, device="cuda").bfloat16()
    side.wait_stream(torch.cuda.current_stream())
    for i in range(40):
        for b in buffers:
            b.fill_(i)
        if i % 2:
            with torch.cuda.stream(side):
                x @ x
        call(None)
        assert all(torch.equal(b, w) for b, w in zip(buffers, want))
    torch.cuda.synchronize()


@pytest.mark.parametrize("new, window", [([4096], 0), ([700, 33, 1200, 801], 0), ([3000, 900], 128), ([41], 0)])
def test_prompts(new, window):
    g = gen(11)
    at, starts = make_starts(new)
    qkv = torch.randn(at[-1], 80, D, generator=g, device="cuda").bfloat16()
    out = torch.empty(at[-1], 64, D, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(at[-1], 64, device="cuda")
    desc = P.layer_desc(window=window)
    repeats(lambda s: P.puzzle_prompt_attn(desc, qkv[:, :64], qkv[:, 64:72], qkv[:, 72:], starts, None, out, lse, stream=s), [out, lse])


@pytest.mark.parametrize("kv", ["fp8", "bf16", "fp4"])
@pytest.mark.parametrize("lens, new, window", [([6000, 5000], [700, 900], 0), ([1300, 2000], [650, 400], 100), ([3000] * 20, [12] * 20, 0),
                                               ([9000], [512], 0)])
def test_chunks(kv, lens, new, window):
    c = Case(kv, lens, new, window, hkv=8)
    repeats(lambda s: P.puzzle_chunk_attn(c.desc, c.view(), c.q, c.starts, c.sinks, c.out, c.lse, workspace=c.workspace, stream=s),
            [c.out, c.lse])
