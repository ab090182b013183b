"""What rows of other sequences, or of none, and earlier launches hold does not change a bit of a sequence's output."""
import math

import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import D, gen, make_starts
from test_gpu_chunk_attn import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [[641], [1202], [333], [35], [641, 1202, 333]])
def test_prompts(new):
    """The rows behind the last sequence, and those of another one."""
    hkv, hq = 8, 64
    at, starts = make_starts(new)
    for others in ([70], [33, 37]):          # belonging to no sequence, then to sequences
        got = []
        for what in (0.0, math.nan, 1e30, -1e4):
            qkv = torch.randn(at[-1] + 70, hq + 2 * hkv, D, generator=gen(3), device="cuda").bfloat16()
            qkv[at[-1]:] = what
            out, lse = torch.empty(at[-1] + 70, hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(at[-1] + 70, hq, device="cuda")
            s = starts if len(others) == 1 else make_starts(new + others)[1]
            P.puzzle_prompt_attn(P.layer_desc(), qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], s, None, out, lse)
            got.append((out[:at[-1]], lse[:at[-1]]))
        for o, l in got[1:]:
            assert torch.equal(l, got[0][1]) and torch.equal(o, got[0][0])


@pytest.mark.parametrize("kv", ["fp8", "bf16", "fp4"])
@pytest.mark.parametrize("lens, new", [([900, 2100], [641, 705]), ([500] * 3, [1, 2, 17]), ([2001] * 20, [1] * 20)])
def test_chunks(kv, lens, new):
    got = []
    for what in (0.0, math.nan, 1e30, -1e4):
        c = Case(kv, lens, new, behind=70, hkv=8)
        c.q[c.at[-1]:] = what
        c.call()
        got.append((c.out[:c.at[-1]], c.lse[:c.at[-1]]))
    for o, l in got[1:]:
        assert torch.equal(l, got[0][1]) and torch.equal(o, got[0][0])


@pytest.mark.parametrize("kv", ["fp8", "bf16", "fp4"])
def test_launches_before(kv):
    """Tensor memory keeps what earlier launches left in it."""
    c = Case(kv, [16 * (i % 40) + 130 + i % 33 for i in range(30)], [1 + i % 3 for i in range(30)], hkv=8)
    got = []
    for scale in (0.0, 1.0, 40.0, -300.0):
        other = Case(kv, [900] * 20, [64] * 20, hkv=8)
        other.q *= scale
        other.call()
        c.call()
        got.append((c.out.clone(), c.lse.clone()))
    for o, l in got[1:]:
        assert torch.equal(l, got[0][1]) and torch.equal(o, got[0][0])
