"""Attention of chunks of new tokens over the paged cache of every type, against the formula in 64 bits."""
import math

import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import BLOCK, D, FLOOR, KINDS, WEIGHT, attention64, cached, check, gen, make_cache, make_starts

pytestmark = pytest.mark.gpu
ALL = ("fp8", "bf16", "fp4")


class Case:
    """Sequences of lens[b] cached tokens, the last new[b] of which are queries."""

    def __init__(self, kv, lens, new, window=0, hkv=2, seed=1, table=True, first=0, behind=0, sinks=True, scales=True,
                 per_seq=None):
        self.kv, self.lens, self.new, self.hkv, self.hq = kv, lens, new, hkv, 8 * hkv
        g = gen(seed)
        self.per_seq = per_seq or max(1, -(-max(lens) // BLOCK))
        nb = len(lens) * self.per_seq + 3
        self.k_cache, self.v_cache = make_cache(kv, nb, hkv, g)
        order = torch.randperm(nb, generator=g, device="cuda") if table else torch.arange(nb, device="cuda")
        self.blocks = order[:len(lens) * self.per_seq].view(len(lens), -1).int().contiguous()
        self.table = self.blocks if table else None
        self.seq_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.k_scale, self.v_scale = ((0.01 + 0.02 * torch.rand(hkv, generator=g, device="cuda")) * (0.3 if kv == "fp4" else 1)
                                      for _ in range(2))
        if not scales:
            self.k_scale = self.v_scale = None
        self.at, self.starts = make_starts(new, first)
        total = self.at[-1] + behind
        self.first = first
        self.q = torch.randn(total, self.hq, D, generator=g, device="cuda").bfloat16()
        self.sinks = torch.randn(self.hq, generator=g, device="cuda") if sinks else None
        self.out = torch.full((total, self.hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((total, self.hq), 7.0, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.desc = P.layer_desc(window=window, kv_dtype=KINDS[kv], num_q_heads=self.hq, num_kv_heads=hkv)
        self.workspace = torch.full((P.puzzle_chunk_attn_workspace_bytes(self.desc, len(lens), total),), 255, dtype=torch.uint8,
                                    device="cuda")

    def view(self):
        return P.kv_view(self.k_cache, self.v_cache, self.seq_lens, block_table=self.table, max_blocks_per_seq=self.per_seq,
                         k_scale=self.k_scale, v_scale=self.v_scale)

    def call(self, q=None):
        P.puzzle_chunk_attn(self.desc, self.view(), self.q if q is None else q, self.starts, self.sinks, self.out, self.lse,
                            workspace=self.workspace, dev_status=self.status)
        torch.cuda.synchronize()
        return self

    def keys(self, b, length, is_v):
        one = torch.ones(self.hkv, device="cuda")
        scale = (self.v_scale if is_v else self.k_scale) if self.k_scale is not None else one
        return cached(self.kv, self.v_cache if is_v else self.k_cache, scale, self.blocks[b], 0, length, is_v)

    def verify(self, status=0):
        assert self.status.item() == status
        for b, n in enumerate(self.new):
            if n:
                rows, m = slice(self.at[b], self.at[b + 1]), min(max(self.lens[b], 0), self.per_seq * BLOCK)
                want, want_lse, size = attention64(self.q[rows], self.keys(b, m, False), self.keys(b, m, True), m - n,
                                                   self.desc.window, self.sinks, self.desc.sm_scale, FLOOR[self.kv])
                check("sequence %d" % b, self.out[rows], self.lse[rows], want, want_lse, size, WEIGHT[self.kv])
        assert (self.out[:self.first] == 7).all() and (self.out[self.at[-1]:] == 7).all()
        assert (self.lse[:self.first] == 7).all() and (self.lse[self.at[-1]:] == 7).all()
        return self


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("lens,new", [([1], [1]), ([17], [1]), ([128], [5]), ([129], [16]), ([1000], [17]), ([777], [333]),
                                      ([2100, 40, 600], [3, 0, 31]), ([300, 300, 1], [300, 1, 1]), ([5000], [2])])
def test_lengths(kv, lens, new):
    Case(kv, lens, new).call().verify()


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("window", [1, 16, 100, 128, 700])
def test_windows(kv, window):
    Case(kv, [900, 50, 2000], [70, 50, 9], window).call().verify()
    Case(kv, [1300, 2000], [650, 400], window, hkv=8).call().verify()      # groups of 32 tokens


@pytest.mark.parametrize("kv", ALL)
def test_wide_groups(kv):
    Case(kv, [1500, 800, 17, 3000], [700, 49, 17, 500], hkv=8).call().verify()


@pytest.mark.parametrize("kv", ALL)
def test_long_context_few_tokens(kv):
    """Keys cut into many parts, some sequences shorter than the parts are many."""
    Case(kv, [20000, 3, 130], [12, 3, 1], hkv=1).call().verify()


@pytest.mark.parametrize("kv", ALL)
def test_many_single_tokens(kv):
    Case(kv, [37 * i % 500 + 1 for i in range(80)], [1] * 80).call().verify()


@pytest.mark.parametrize("kv", ALL)
def test_no_table_no_sinks_no_scales(kv):
    Case(kv, [200, 90], [20, 90], table=False, sinks=False, scales=False).call().verify()


def test_rows_of_no_sequence_stay():
    Case("fp8", [200, 90], [20, 90], first=3, behind=40).call().verify()
    Case("fp8", [200, 9000], [20, 4], first=3, behind=40, hkv=1).call().verify()


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("hkv", [1, 8])
def test_more_tokens_than_the_sequence_has(kv, hkv):
    """Positions below zero see nothing: zeros, and the sink's own log sum."""
    c = Case(kv, [5, 0, 400], [20, 7, 2], hkv=hkv).call().verify()
    assert (c.out[:15] == 0).all() and (c.out[20:27] == 0).all()
    assert torch.equal(c.lse[20:27], c.sinks.expand(7, -1).contiguous()) or (c.lse[20:27] - c.sinks).abs().max() < 1e-5
    c = Case(kv, [5, 0, 400], [20, 7, 2], hkv=hkv, sinks=False).call().verify()
    assert (c.lse[20:27] == -math.inf).all()


def test_sequence_longer_than_its_table_row():
    Case("fp8", [1000, 100], [6, 6], per_seq=20).call().verify(status=P.DEV_SEQ_TOO_LONG)


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_bad_block_counts_as_zeros(kv, bad):
    c = Case(kv, [400, 200], [30, 5])
    lost = c.blocks[0, 7].item()
    spare = c.k_cache.shape[0] - 1
    spare = next(i for i in range(c.k_cache.shape[0]) if i not in set(c.blocks.flatten().tolist()))
    c.k_cache[spare] = 0
    c.v_cache[spare] = 0
    right = c.blocks.clone()
    right[0, 7] = spare
    c.table = c.blocks.clone()
    c.table[0, 7] = bad
    c.blocks = right
    c.call().verify(status=P.DEV_BAD_BLOCK)
    assert lost != spare


@pytest.mark.parametrize("starts", [[0, 10, 5], [-3, 10, 20], [0, 10, 99]])
def test_bad_starts_skip_the_sequence(starts):
    c = Case("fp8", [100, 200], [10, 10])
    c.starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    c.call()
    assert c.status.item() == P.DEV_BAD_STARTS
    if starts[0] == 0:      # the other one is served
        want, want_lse, size = attention64(c.q[:10], c.keys(0, 100, False), c.keys(0, 100, True), 90, 0, c.sinks, 0.125, FLOOR["fp8"])
        check("sequence 0", c.out[:10], c.lse[:10], want, want_lse, size, WEIGHT["fp8"])


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("window", [0, 40])
def test_nan_in_values_that_a_row_does_not_see(kv, window):
    """In unused slots of the last block, in the chunk itself, before the window, and where all rows see it."""
    for hkv, lens, new in ((2, [500, 90], [45, 33]), (8, [1600, 500], [700, 300])):
        c = Case(kv, lens, new, window, hkv=hkv)
        for b, pos in ((0, lens[0] - 20), (0, lens[0] - new[0] - 41), (0, 3), (1, lens[1] - 1)):
            blk, slot = c.blocks[b, pos // BLOCK].item(), pos % BLOCK
            if kv == "bf16":
                c.v_cache[blk, 0, slot, 9] = math.nan
                c.v_cache[blk, 1, slot, 30] = -math.inf
            elif kv == "fp8":
                c.v_cache[blk, 0, slot, 9] = 0x7f
                c.v_cache[blk, 1, slot, 30] = 0xff
            else:
                c.v_cache[blk, 0, 512 + 16 * 1 + 4 * (slot % 8 // 2) + 2 * (slot // 8) + slot % 2] = 0x7f
        for b in (0, 1):                     # behind the sequence's end
            for pos in range(lens[b], -(-lens[b] // BLOCK) * BLOCK):
                blk, slot = c.blocks[b, pos // BLOCK].item(), pos % BLOCK
                if kv == "bf16":
                    c.v_cache[blk, :, slot] = math.nan
                    c.k_cache[blk, :, slot] = math.nan
                elif kv == "fp8":
                    c.v_cache[blk, :, slot] = 0x7f
                    c.k_cache[blk, :, slot] = 0x7f
        c.call().verify()


@pytest.mark.parametrize("kv", ["fp8", "fp4"])
def test_weights_far_below_the_largest_one(kv):
    """One key with a weight of 1 and thousands of 2^-22 each: they keep their bits."""
    c = Case(kv, [9000], [16], hkv=1, sinks=False)
    c.q.zero_()
    c.q[:, :, 0] = 8.0
    c.k_cache.zero_()
    blk = c.blocks[0, 0].item()
    c.k_scale.fill_(0.25)
    c.v_scale.fill_(1.0)
    value = 15.25                                   # logit of the one key, in natural units: 2^-22 for all others
    c.desc.sm_scale = value / (8.0 * 4.0 * 0.25)
    if kv == "fp8":
        c.k_cache[blk, 0, 0, 0] = 0x48              # 4.0
        c.v_cache.fill_(0x38)                       # 1.0
        c.v_cache[blk, 0, 0] = 0                    # the one key has no value: all of the output is the others'
    else:
        c.k_cache[:, :, 512:] = 0x38
        c.k_cache[blk, 0, 0] = 0x06                 # 4.0 in channel 0
        c.v_cache[:, :, :512] = 0x22                # 1.0
        c.v_cache[:, :, 512:] = 0x38
        c.v_cache[blk, 0, 0:32] = 0x20
        c.v_cache[blk, 0, 256:288] = 0x20
    c.call().verify()


def test_strided_queries():
    c = Case("fp8", [300, 100], [40, 13])
    wide = torch.randn(53, c.hq + 7, D, device="cuda").bfloat16()
    wide[:, 3:3 + c.hq] = c.q
    c.call(wide[:, 3:3 + c.hq]).verify()


def test_the_same_bits_twice_and_on_another_stream():
    c = Case("fp4", [5000, 100], [40, 13]).call()
    out, lse = c.out.clone(), c.lse.clone()
    other = torch.cuda.Stream()
    c.out.fill_(3)
    c.workspace.fill_(255)
    torch.cuda.synchronize()
    P.puzzle_chunk_attn(c.desc, c.view(), c.q, c.starts, c.sinks, c.out, c.lse, workspace=c.workspace, stream=other)
    torch.cuda.synchronize()
    assert torch.equal(out, c.out) and torch.equal(lse, c.lse)


def test_graph_with_growing_sequences():
    """A captured call follows the lengths and starts that its tensors hold at replay."""
    c = Case("fp8", [3000, 700], [9, 40])
    c.call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.puzzle_chunk_attn(c.desc, c.view(), c.q, c.starts, c.sinks, c.out, c.lse, workspace=c.workspace, dev_status=c.status)
    for lens, new in (([2500, 699], [30, 19]), ([17, 500], [1, 48]), ([3000, 700], [0, 49])):
        c.lens, c.new = lens, new
        c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.at, starts = make_starts(new)
        c.starts.copy_(starts)
        graph.replay()
        torch.cuda.synchronize()
        c.verify()


def test_agrees_with_the_multi_token_kernel():
    c = Case("fp8", [900, 333, 4000], [4, 4, 4], hkv=8).call()
    ws = torch.empty(P.puzzle_decode_attn_tokens_workspace_bytes(c.desc, 3, 4), dtype=torch.uint8, device="cuda")
    P.puzzle_decode_attn_tokens_workspace_init(c.desc, 3, 4, ws)
    out = torch.empty(3, 4, c.hq, D, dtype=torch.bfloat16, device="cuda")
    P.puzzle_decode_attn_tokens(c.desc, c.view(), c.q.view(3, 4, c.hq, D), c.sinks, out, workspace=ws)
    # both are rounded to bf16, each by at most 2^-8 of its value; their weights are off by 2^-11 and less
    a, b = out.view_as(c.out).double(), c.out.double()
    assert ((a - b).abs() <= 2.0 ** -7 * b.abs() + 2e-3).all()
