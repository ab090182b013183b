"""A decode step with rotation over a context that is dealt to several ranks, one rank after the other on one GPU: only the owner
of the newest block stores the token, every rank gets the rotated query."""
import numpy as np
import pytest
import torch

import kv_reference as R
from helpers import bf16_bits
from test_gpu_kv_rope import KINDS, Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("world", [2, 3])
def test_the_recipe_of_context_slice(kind, world):
    import paper_2602_11937_b200 as P
    s = Setup(KINDS[kind], [144, 1, 0, 16, 17, 97, 33], 1, seed=world)
    s.upload()
    q, k, v = s.parts(s.d["qkv"])
    lens = s.d["lens"]
    offset = torch.clamp(lens - 1, min=0)
    scratch = [torch.zeros(s.batch, *t.shape[1:], dtype=t.dtype, device="cuda") for t in (s.d["k"], s.d["v"])]
    one = torch.clamp(lens, max=1)
    place = P.kv_view(*scratch, one, max_blocks_per_seq=1, k_scale=s.d["ks"], v_scale=s.d["vs"])
    rotated = []
    for rank in range(world):
        _, append = P.context_slice(lens, rank, world)
        table = s.d["table"][:, rank::world].contiguous()
        view = P.kv_view(s.d["k"], s.d["v"], append, block_table=table, k_scale=s.d["ks"], v_scale=s.d["vs"])
        q_out = s.dead((s.batch, 1, s.hq, 64))
        P.puzzle_kv_append_rope(s.desc, place, P.rope_view(s.d["cs"], pos_offset=offset), q, k, v, q_out,
                                dev_status=s.d["status"])
        P.puzzle_kv_append_rope(s.desc, view, P.rope_view(s.d["cs"], pos_offset=lens - append), None, k, v,
                                dev_status=s.d["status"])
        rotated.append(q_out)
    torch.cuda.synchronize()
    hq, hk, hv = (bf16_bits(x) for x in s.parts(s.qkv))
    want = R.append(s.ref, s.table, s.max_blocks, s.lens, None, hq, hk, hv, s.k_scale, s.v_scale, s.cos_sin, s.rotary, False, None)
    for q_out in rotated:
        assert np.array_equal(bf16_bits(q_out), want)
    s.check_cache()
    assert int(s.d["status"].item()) == 0
