"""Append of packed tokens: the bytes that the rectangular append writes, the rotated rows it gives out, and the rows and slots
that it leaves alone."""
import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import BLOCK, D, KINDS, gen, make_cache, make_starts

pytestmark = pytest.mark.gpu
ALL = ("fp8", "bf16", "fp4")


class Case:
    def __init__(self, kv, lens, new, hkv=3, seed=1, rotary=64, interleaved=False, offset=None, first=0, behind=0, per_seq=None,
                 positions=4096):
        self.kv, self.lens, self.new, self.hkv, self.hq = kv, lens, new, hkv, 8 * hkv
        g = gen(seed)
        self.per_seq = per_seq or max(1, -(-max(lens) // BLOCK))
        nb = len(lens) * self.per_seq + 2
        self.caches = make_cache(kv, nb, hkv, g)
        self.table = torch.randperm(nb, generator=g, device="cuda")[:len(lens) * self.per_seq].view(len(lens), -1).int().contiguous()
        self.seq_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.scales = [0.01 + 0.02 * torch.rand(hkv, generator=g, device="cuda") for _ in range(2)]
        self.at, self.starts = make_starts(new, first)
        self.total = self.at[-1] + behind
        self.qkv = torch.randn(self.total, self.hq + 2 * hkv, D, generator=g, device="cuda").bfloat16()
        self.cos_sin = torch.rand(positions, rotary, generator=g, device="cuda") * 2 - 1
        self.offset = None if offset is None else torch.tensor(offset, dtype=torch.int32, device="cuda")
        self.rope = P.rope_view(self.cos_sin, interleaved=interleaved, pos_offset=self.offset)
        self.desc = P.layer_desc(kv_dtype=KINDS[kv], num_q_heads=self.hq, num_kv_heads=hkv)
        self.q_out = torch.full((self.total, self.hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.k_out = torch.full((self.total, hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def parts(self):
        return self.qkv[:, :self.hq], self.qkv[:, self.hq:self.hq + self.hkv], self.qkv[:, self.hq + self.hkv:]

    def view(self, caches=None):
        k, v = caches or self.caches
        return P.kv_view(k, v, self.seq_lens, block_table=self.table, k_scale=self.scales[0], v_scale=self.scales[1])

    def call(self, rotate=True, with_q=True, with_k=True, keep_last=0):
        q, k, v = self.parts()
        if rotate:
            P.puzzle_kv_append_packed(self.desc, self.view(), self.rope, q if with_q else None, k, v, self.starts,
                                      self.q_out if with_q else None, self.k_out if with_k else None, keep_last,
                                      dev_status=self.status)
        else:
            P.puzzle_kv_append_packed(self.desc, self.view(), None, None, k, v, self.starts, keep_last=keep_last, dev_status=self.status)
        torch.cuda.synchronize()

    def rectangle(self, caches, rotate=True):
        """The same tokens through the rectangular entry points, into `caches`: the rotated queries."""
        n = max(max(self.new), 1)
        box = torch.zeros(len(self.new), n, self.hq + 2 * self.hkv, D, dtype=torch.bfloat16, device="cuda")
        for b, m in enumerate(self.new):
            box[b, :m] = self.qkv[self.at[b]:self.at[b] + m]
        lens = torch.tensor(self.new, dtype=torch.int32, device="cuda")
        q, k, v = box[:, :, :self.hq], box[:, :, self.hq:self.hq + self.hkv], box[:, :, self.hq + self.hkv:]
        out = torch.full((len(self.new), n, self.hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        if rotate:
            P.puzzle_kv_append_rope(self.desc, self.view(caches), self.rope, q, k, v, out, new_lens=lens)
        else:
            P.puzzle_kv_append_tokens(self.desc, self.view(caches), k.contiguous(), v.contiguous(), new_lens=lens)
        torch.cuda.synchronize()
        return out

    def turned(self, rows, positions, heads):
        """Rows [n][heads][D] rotated, float32, every product and sum rounded on its own."""
        r = self.cos_sin.shape[1]
        half = r // 2
        row = self.cos_sin[positions][:, None]
        c, s = row[..., :half], row[..., half:]
        x = rows.float()
        y = x.clone()
        i, j = (slice(0, r, 2), slice(1, r, 2)) if self.rope.interleaved else (slice(0, half), slice(half, r))
        y[..., i] = x[..., i] * c - x[..., j] * s
        y[..., j] = x[..., j] * c + x[..., i] * s
        return y


def same_bytes(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("rotary,interleaved", [(64, False), (64, True), (48, False), (16, True), (None, False)])
def test_the_bytes_of_the_rectangular_append(kv, rotary, interleaved):
    c = Case(kv, [70, 1, 500, 33, 18], [70, 1, 130, 0, 5], rotary=rotary or 64, interleaved=interleaved)
    want = [x.clone() for x in c.caches]
    out = c.rectangle(want, rotary is not None)
    c.call(rotary is not None)
    assert c.status.item() == 0 and same_bytes(c.caches, want)
    if rotary is not None:
        for b, n in enumerate(c.new):
            rows = slice(c.at[b], c.at[b + 1])
            assert torch.equal(c.q_out[rows], out[b, :n])
            pos = torch.arange(c.lens[b] - n, c.lens[b], device="cuda")
            assert torch.equal(c.k_out[rows], c.turned(c.parts()[1][rows], pos, c.hkv).bfloat16())


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("lens,new", [([1], [1]), ([32], [32]), ([35], [32]), ([131], [33]), ([64] * 70, [1] * 70),
                                      ([3, 200, 77] * 25, [3, 64, 0] * 25), ([2050], [2047])])
def test_lengths(kv, lens, new):
    c = Case(kv, lens, new, hkv=1)
    want = [x.clone() for x in c.caches]
    c.rectangle(want)
    c.call()
    assert same_bytes(c.caches, want)


def test_heads_beyond_a_group_of_eight():
    c = Case("fp4", [90, 40], [33, 40], hkv=11)
    want = [x.clone() for x in c.caches]
    c.rectangle(want)
    c.call()
    assert same_bytes(c.caches, want)


@pytest.mark.parametrize("with_q,with_k", [(False, True), (True, False), (False, False)])
def test_without_queries_or_keys_out(with_q, with_k):
    c = Case("fp8", [90, 40], [33, 40])
    want = [x.clone() for x in c.caches]
    c.rectangle(want)
    c.call(with_q=with_q, with_k=with_k)
    assert same_bytes(c.caches, want)
    assert with_q or (c.q_out == 7).all()
    assert with_k or (c.k_out == 7).all()


def test_rows_of_no_sequence_stay():
    c = Case("bf16", [90, 40], [33, 40], first=6, behind=50)
    c.call()
    for x in (c.q_out, c.k_out):
        assert (x[:6] == 7).all() and (x[79:] == 7).all() and not (x[6:79] == 7).all()


def test_offsets_and_positions_beyond_the_table():
    c = Case("fp8", [90, 40, 60], [33, 40, 60], offset=[100, -5, 0], positions=160)
    before = [x.clone() for x in c.caches]
    c.rectangle(before)
    c.call()
    assert c.status.item() == P.DEV_BAD_POSITION and same_bytes(c.caches, before)
    assert (c.q_out[33:38] == 7).all() and (c.k_out[33:38] == 7).all()       # positions -5 .. -1
    # positions 57 + 100 .. 89 + 100 of a table of 160: the first three tokens are rotated, the others left out
    assert (c.q_out[:3] != 7).any(-1).any(-1).all() and (c.q_out[3:33] == 7).all()


@pytest.mark.parametrize("kv", ALL)
def test_more_tokens_than_the_sequence_has(kv):
    c = Case(kv, [5, 0, 40], [20, 7, 2])
    want = [x.clone() for x in c.caches]
    c.rectangle(want)
    c.call()
    assert same_bytes(c.caches, want) and c.status.item() == 0
    assert (c.q_out[:15] == 7).all() and (c.k_out[20:27] == 7).all()


def test_long_sequences_and_bad_blocks():
    c = Case("fp8", [400, 100], [6, 50], per_seq=20)
    before = [x.clone() for x in c.caches]
    c.table[1, 4] = 10 ** 6                     # positions 64 .. 79
    c.rectangle(before)
    c.call()
    assert c.status.item() == P.DEV_SEQ_TOO_LONG | P.DEV_BAD_BLOCK and same_bytes(c.caches, before)
    assert (c.q_out[:6] == 7).all()
    rows = slice(6, 56)                         # the rows go out whatever the table says
    assert torch.equal(c.k_out[rows], c.turned(c.parts()[1][rows], torch.arange(50, 100, device="cuda"), 3).bfloat16())


@pytest.mark.parametrize("starts", [[0, 33, 20], [-1, 33, 73], [0, 33, 74]])
def test_bad_starts_skip_the_sequence(starts):
    c = Case("fp8", [90, 40], [33, 40])
    before = [x.clone() for x in c.caches]
    c.starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    c.call()
    assert c.status.item() == P.DEV_BAD_STARTS
    bad = 0 if starts[0] < 0 else 1
    for x, y in zip(c.caches, before):
        assert torch.equal(x[c.table[bad].long()], y[c.table[bad].long()])


def test_in_place():
    c = Case("fp8", [90, 40], [33, 40])
    c.call()
    q, k = (x.contiguous() for x in c.parts()[:2])
    P.puzzle_kv_append_packed(c.desc, c.view(), c.rope, q, k, c.parts()[2], c.starts, q, k)
    torch.cuda.synchronize()
    assert torch.equal(q, c.q_out) and torch.equal(k, c.k_out)


def test_no_tokens_at_all():
    c = Case("fp8", [90, 40], [0, 0])
    before = [x.clone() for x in c.caches]
    c.call()
    P.puzzle_prompt_attn(c.desc, *c.parts(), c.starts, None, c.q_out)
    ws = torch.empty(P.puzzle_chunk_attn_workspace_bytes(c.desc, 2, 0), dtype=torch.uint8, device="cuda")
    P.puzzle_chunk_attn(c.desc, c.view(), c.parts()[0], c.starts, None, c.q_out, workspace=ws)
    torch.cuda.synchronize()
    assert same_bytes(c.caches, before)


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("keep", [1, 16, 31, 500])
def test_only_the_last_tokens_are_kept(kv, keep):
    c = Case(kv, [70, 1, 500, 33, 18], [70, 1, 130, 0, 5])
    before = [x.clone() for x in c.caches]
    c.rectangle(before)                          # all of them, then what was there before in the places that are left alone
    was = [x.clone() for x in c.caches]
    new, lens = list(c.new), list(c.lens)
    for b, n in enumerate(new):                  # the same bytes by appending the tail alone
        if n > keep:
            for p in range(lens[b] - n, lens[b] - keep):
                blk, t = c.table[b, p // BLOCK].item(), p % BLOCK
                for x, y, is_v in zip(before, was, (False, True)):
                    if kv != "fp4":
                        x[blk, :, t] = y[blk, :, t]
                        continue
                    d = torch.arange(D, device="cuda")
                    byte = 256 * (d // 32) + 32 * (t // 2) + d % 32 if is_v else 32 * t + d // 2
                    odd = torch.full_like(d, t % 2) if is_v else d % 2
                    for e in (0, 1):
                        at, mask = byte[odd == e], (0xf0 if e else 0x0f)
                        x[blk, :, at] = (x[blk, :, at] & (0xff ^ mask)) | (y[blk, :, at] & mask)
                    g = torch.arange(4, device="cuda")
                    at = 512 + 16 * g + (4 * (t % 8 // 2) + 2 * (t // 8) + t % 2 if is_v else 2 * (t % 8) + t // 8)
                    x[blk, :, at] = y[blk, :, at]
    c.call(keep_last=keep)
    assert c.status.item() == 0 and same_bytes(c.caches, before)
    for b, n in enumerate(new):
        rows, pos = slice(c.at[b], c.at[b + 1]), torch.arange(lens[b] - n, lens[b], device="cuda")
        assert torch.equal(c.k_out[rows], c.turned(c.parts()[1][rows], pos, c.hkv).bfloat16())
        assert torch.equal(c.q_out[rows], c.turned(c.parts()[0][rows], pos, c.hq).bfloat16())
