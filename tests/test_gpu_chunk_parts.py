"""Chunk attention whose keys are cut into parts: what is tested elsewhere in one piece, here with a merge behind it.  That a call is cut
shows in its launches."""
import math

import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import BLOCK, make_starts
from test_gpu_chunk_attn import Case

pytestmark = pytest.mark.gpu
ALL = ("fp8", "bf16", "fp4")


def cut(c, status=0):
    before = P.puzzle_launch_count()
    c.call()
    assert P.puzzle_launch_count() - before == 2, "not cut"
    return c.verify(status)


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("hkv, lens, new", [(8, [9000], [5]), (8, [2100], [1]), (1, [16384], [5]), (1, [65536], [3]), (8, [32768], [18]),
                                            (1, [80000], [7]), (2, [9000, 3000], [2, 1]), (1, [20000, 3, 130], [12, 3, 1]),
                                            (8, [20000], [64]), (8, [12000], [150]), (8, [30000], [512])])
def test_lengths(kv, hkv, lens, new):
    cut(Case(kv, lens, new, hkv=hkv))


@pytest.mark.parametrize("kv", ALL)
def test_short_sequences_beside_a_long_one(kv):
    """More parts than the short ones have tiles, or keys."""
    cut(Case(kv, [20000, 1, 17, 129, 0, 2000], [3, 1, 9, 4, 0, 2], hkv=1))
    cut(Case(kv, [300, 5], [5, 5], hkv=8, per_seq=4096))


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("window", [5000, 3000])
def test_windows(kv, window):
    cut(Case(kv, [9000, 700], [5, 9], window, hkv=1))


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("sinks", [True, False])
def test_positions_below_zero(kv, sinks):
    c = cut(Case(kv, [20000, 5, 0], [4, 20, 7], hkv=1, sinks=sinks))
    assert (c.out[4:19] == 0).all() and (c.out[24:31] == 0).all()
    if sinks:
        assert (c.lse[24:31] - c.sinks).abs().max() < 1e-5
    else:
        assert (c.lse[24:31] == -math.inf).all()


@pytest.mark.parametrize("kv", ALL)
def test_rows_of_no_sequence_stay(kv):
    cut(Case(kv, [20000, 9000], [20, 4], first=3, behind=40, hkv=1))


@pytest.mark.parametrize("kv", ALL)
def test_no_table_no_sinks_no_scales(kv):
    cut(Case(kv, [9000, 5000], [5, 2], table=False, sinks=False, scales=False, hkv=1))


def test_sequence_longer_than_its_table_row():
    cut(Case("fp8", [9000, 100], [6, 6], per_seq=500, hkv=1), status=P.DEV_SEQ_TOO_LONG)


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_bad_blocks_count_as_zeros(kv, bad):
    c = Case(kv, [9000], [5], hkv=8)
    spare = sorted(set(range(c.k_cache.shape[0])) - set(c.blocks.flatten().tolist()))[0]
    c.k_cache[spare] = 0
    c.v_cache[spare] = 0
    right, c.table = c.blocks.clone(), c.blocks.clone()
    for j in (0, 100, 101, 562):
        right[0, j] = spare
        c.table[0, j] = bad
    c.blocks = right
    cut(c, status=P.DEV_BAD_BLOCK)


@pytest.mark.parametrize("kv", ALL)
def test_nan_in_values_and_keys(kv):
    """In a value that all rows see, in one that only some see, and in keys behind the end; then in a key of one part."""
    c = Case(kv, [9000], [5], hkv=8)
    for pos in (4000, 8997):
        blk, slot = c.blocks[0, pos // BLOCK].item(), pos % BLOCK
        if kv == "bf16":
            c.v_cache[blk, 0, slot, 9] = math.nan
            c.v_cache[blk, 1, slot, 30] = -math.inf
        elif kv == "fp8":
            c.v_cache[blk, 0, slot, 9] = 0x7f
        else:
            c.v_cache[blk, 0, 512 + 16 + 4 * (slot % 8 // 2) + 2 * (slot // 8) + slot % 2] = 0x7f
    for pos in range(9000, 9008):
        blk, slot = c.blocks[0, pos // BLOCK].item(), pos % BLOCK
        if kv != "fp4":
            c.k_cache[blk, :, slot] = math.nan if kv == "bf16" else 0x7f
            c.v_cache[blk, :, slot] = math.nan if kv == "bf16" else 0x7f
    cut(c)
    blk = c.blocks[0, 6000 // BLOCK].item()
    if kv == "fp4":
        c.k_cache[blk, 2, 512] = 0x7f
    else:
        c.k_cache[blk, 2, 0, 5] = math.nan if kv == "bf16" else 0x7f
    c.call()
    heads = torch.arange(c.hq, device="cuda") // 8 == 2
    assert c.out[:, heads].isnan().all() and c.lse[:, heads].isnan().all()
    assert not c.lse[:, ~heads].isnan().any()


@pytest.mark.parametrize("kv", ALL)
def test_many_entries_of_starts(kv):
    """The merge finds a row's sequence among many, most of them empty."""
    lens, new = [20000 if b in (0, 17, 299) else 40 for b in range(300)], [0] * 300
    for b, n in ((0, 3), (16, 1), (17, 5), (31, 1), (32, 2), (200, 1), (299, 4)):
        new[b] = n
    cut(Case(kv, lens, new, hkv=1, per_seq=1250))


def test_graph_follows_lengths_and_starts():
    c = Case("fp8", [20000, 9000], [9, 40], hkv=1)
    cut(c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.puzzle_chunk_attn(c.desc, c.view(), c.q, c.starts, c.sinks, c.out, c.lse, workspace=c.workspace, dev_status=c.status)
    for lens, new in (([100, 15000], [30, 19]), ([17, 500], [1, 48]), ([20000, 9000], [0, 49])):
        c.lens, c.new = lens, new
        c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.at, starts = make_starts(new)
        c.starts.copy_(starts)
        c.workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        c.verify()
