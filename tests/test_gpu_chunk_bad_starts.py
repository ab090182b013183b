"""Bad entries of starts in calls whose keys are cut into parts: only the sequence they belong to is skipped."""
import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import FLOOR, WEIGHT, attention64, check
from test_gpu_chunk_attn import Case

pytestmark = pytest.mark.gpu

# (starts, the sequences that are valid)
STARTS = [([0, 12, 99, 12, 24], [0, 3]), ([0, 5, -1, 5, 10], [0, 3]), ([10, 22, 0, 10, 10], [0, 2]), ([0, 99, 5, 8, 20], [2, 3]),
          ([0, 2, 99, 2, 6], [0, 3]), ([3, 3, 24, 24, 2], [1]), ([-1, -1, -1, -1, 24], []), ([24, 12, 8, 4, 0], [])]


@pytest.mark.parametrize("kv", ["fp8", "bf16", "fp4"])
@pytest.mark.parametrize("starts, valid", STARTS)
def test_valid_sequences_are_served(kv, starts, valid):
    c = Case(kv, [20000, 19000, 300, 20], [6, 6, 6, 6], hkv=1)
    c.starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    before = P.puzzle_launch_count()
    c.call()
    assert P.puzzle_launch_count() - before == 2                # the keys are cut
    assert c.status.item() == P.DEV_BAD_STARTS
    left = torch.ones(24, dtype=torch.bool, device="cuda")
    for b in valid:
        rows, m = slice(starts[b], starts[b + 1]), c.lens[b]
        left[rows] = False
        n = starts[b + 1] - starts[b]
        want, lse, size = attention64(c.q[rows], c.keys(b, m, False), c.keys(b, m, True), m - n, 0, c.sinks, c.desc.sm_scale, FLOOR[kv])
        check("sequence %d" % b, c.out[rows], c.lse[rows], want, lse, size, WEIGHT[kv])
    assert (c.out[left] == 7).all() and (c.lse[left] == 7).all()
