"""Decode attention over the 4-bit cache against the float64 oracle on the same bytes.

Bound on the error of one output, derived from the kernel's roundings.  V is exact; a weight is off by 2^-11 of itself
(its f16 rounding) plus 2^-25 of the reference maximum (f16 subnormals); logits are sums of 64 exact products in
float32, off by at most 64 * 2^-24 = 2^-18 of the sum of the products' magnitudes, which for the inputs here (|q|, |k|
below 5, sm_scale 1/8) stays below 64 * 25 / 8 = 200 in the worst case and near 10 in earnest: 2^-14.7 of a weight,
in the numerator and in the normaliser.  ex2 and the merges add 2^-20.  So 2^-11 + 2 * 2^-14.7 + 2^-20 < 2^-10 of
A = sum p |v| / Z (computed by the oracle on |V|), plus N 2^-25 max |v|, plus the output's own rounding, 2^-8 of it."""
import numpy as np
import pytest
import torch

import oracle
from helpers import bf16_bits, bits_to_bf16
import kv_reference as R

pytestmark = pytest.mark.gpu


def value_bound(ref, mag, keys, vmax, bf16=True):
    return (2.0 ** -8 * np.abs(ref) if bf16 else 0.0) + 2.0 ** -10 * mag + (keys + 1) * 2.0 ** -25 * vmax


class Case:
    """Random 4-bit caches, permuted table, ragged lengths; what no query may see holds NaN scales."""

    def __init__(self, lens, hkv=2, max_blocks=None, paged=True, seed=0, window=0, poison=True, n_q=1, q_lens=None,
                 scale=1.0, sinks=True):
        import paper_2602_11937_b200 as P
        self.P, self.hkv, self.hq, self.window, self.n_q = P, hkv, 8 * hkv, window, n_q
        self.lens = np.asarray(lens, np.int32)
        self.q_lens = None if q_lens is None else np.asarray(q_lens, np.int32)
        self.batch = len(lens)
        self.mb = max_blocks or max(1, -(-max(lens) // 16))
        r = np.random.default_rng(seed)
        nb = self.batch * self.mb + (3 if paged else 0)
        self.table = r.permutation(nb)[:self.batch * self.mb].reshape(self.batch, -1).astype(np.int32) if paged else None
        self.k, self.v = R.fp4_random_cache(nb, hkv, seed + 1, scale)
        self.k_scale, self.v_scale = ((0.7 + 0.6 * r.random(hkv)).astype(np.float32) for _ in range(2))
        q = torch.randn(self.batch, n_q, self.hq, 64, generator=torch.Generator().manual_seed(seed)).clamp(-4, 4)
        self.q = q.to(torch.bfloat16)
        self.sinks = r.standard_normal(self.hq).astype(np.float32) if sinks else None
        if poison:
            for b in range(self.batch):
                seen = [i for i in range(self.mb * 16) if i < self.lens[b] and
                        (not window or i >= self.lens[b] - n_q + 1 - window)]
                lo, hi = (seen[0], seen[-1] + 1) if seen else (0, 0)
                for t in [*range(lo // 16 * 16, lo), *range(hi, -(-max(hi, 1) // 16) * 16)]:
                    blk = b * self.mb + t // 16 if self.table is None else self.table[b, t // 16]
                    for s in range(4):
                        self.k[blk, :, R.k_scale_at(t % 16, s)] = 0x7F
                        self.v[blk, :, R.v_scale_at(t % 16, s)] = 0xFF

    def upload(self):
        up = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.d = {n: up(getattr(self, n)) for n in ("k", "v", "table", "lens", "k_scale", "v_scale", "sinks", "q_lens")}
        self.d["q"] = self.q.cuda()
        self.desc = self.P.layer_desc(window=self.window, kv_dtype=self.P.KV_FP4_E2M1, num_q_heads=self.hq,
                                      num_kv_heads=self.hkv)
        self.view = self.P.kv_view(self.d["k"], self.d["v"], self.d["lens"], block_table=self.d["table"],
                                   max_blocks_per_seq=self.mb, k_scale=self.d["k_scale"], v_scale=self.d["v_scale"])
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        return self

    def oracle(self, token=0, lens=None, absolute=False):
        """(out, lse) of query token `token` as a decode step of its own."""
        if lens is None:
            ql = np.full(self.batch, self.n_q) if self.q_lens is None else np.clip(self.q_lens, 0, self.n_q)
            lens = np.where(token < ql, np.maximum(self.lens - ql + token + 1, 0), 0).astype(np.int32)
        table = self.table
        if table is not None:      # out-of-range entries of blocks nobody sees
            table = np.clip(table, 0, self.k.shape[0] - 1)
        v = self.v.copy()
        if absolute:
            v[:, :, :512] &= 0x77
        out, lse = oracle.decode_attn(self.k, v, R.FP4, table, self.mb, lens, self.k_scale, self.v_scale,
                                      bf16_bits(self.q[:, token].contiguous()), self.sinks, self.window, 0.125)
        return out.reshape(self.batch, self.hq, 64), lse.reshape(self.batch, self.hq)

    def check(self, got, got_lse, token=0, bf16=True, lens=None, rows=None):
        ref, lse = self.oracle(token, lens)
        mag, _ = self.oracle(token, lens, absolute=True)
        rows = slice(None) if rows is None else rows
        got, got_lse, ref, lse, mag = got[rows], got_lse[rows], ref[rows], lse[rows], mag[rows]
        assert not np.isnan(got).any()
        scales = R.E4M3[self.v[:, :, 512:]]
        vmax = 6.0 * float(np.nanmax(np.abs(scales))) * float(self.v_scale.max())
        bound = value_bound(ref, mag, int(self.lens.max()), vmax, bf16)
        assert (np.abs(got - ref) <= bound).all(), float((np.abs(got - ref) - bound).max())
        fin = np.isfinite(lse)
        assert np.array_equal(np.isfinite(got_lse), fin) and np.array_equal(got_lse[~fin], lse[~fin])
        # logits off by 2^-18 * 200 at the very worst, 1e-4 in earnest (as for the other caches)
        assert (np.abs(got_lse[fin] - lse[fin]) <= 1e-4).all()

    def run(self, splits=0, ws=None, call=None):
        P = self.P
        if ws is None:
            ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(self.desc, self.batch, splits), dtype=torch.uint8,
                             device="cuda").fill_(0xFF)
            P.puzzle_decode_attn_workspace_init(self.desc, self.batch, ws)
        out = torch.full((self.batch, self.hq, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.batch, self.hq), float("nan"), device="cuda")
        P.puzzle_decode_attn(self.desc, self.view, self.d["q"][:, 0].contiguous(), self.d["sinks"], out, lse,
                             num_splits=splits, workspace=ws, dev_status=self.status)
        torch.cuda.synchronize()
        return out.double().cpu().numpy(), lse.double().cpu().numpy()


LENS = [700, 1, 0, 16, 17, 333, 64, 65, 2, 1500]


@pytest.mark.parametrize("splits", [0, -1, -2, 1, 2, 5, 17])
@pytest.mark.parametrize("window", [0, 1, 15, 100, 128, 600])
def test_ragged_lengths_every_schedule(window, splits):
    c = Case(LENS, window=window, seed=window).upload()
    c.check(*c.run(splits))
    assert int(c.status.item()) == 0


@pytest.mark.parametrize("hkv", [1, 3, 8])
@pytest.mark.parametrize("splits", [0, -1, -2, 3])
def test_head_counts_without_sinks(hkv, splits):
    c = Case([130, 0, 257, 48], hkv=hkv, paged=hkv != 3, sinks=False, seed=hkv).upload()
    c.check(*c.run(splits))


@pytest.mark.parametrize("length", list(range(1, 20)) + [31, 32, 33, 47, 48, 63, 64, 65, 127, 128, 129, 191, 192, 193, 256])
def test_every_edge_of_a_block_and_a_tile(length):
    for splits in (0, -1, -2):
        c = Case([length, max(0, length - 1)], hkv=1, max_blocks=20, seed=length).upload()
        c.check(*c.run(splits))


@pytest.mark.parametrize("splits", [0, -1])
def test_long_context_many_ctas(splits):
    c = Case([20001, 13333], hkv=2, seed=3).upload()
    c.check(*c.run(splits))


def test_many_short_pairs():
    """More pairs than the narrow-window kernel takes (one warp per pair), and a batch beyond the CTA-balanced kernel's."""
    r = np.random.default_rng(0)
    c = Case(list(r.integers(0, 130, size=300)), hkv=4, window=100, seed=5, max_blocks=9).upload()
    c.check(*c.run(0))
    c = Case(list(r.integers(0, 40, size=1100)), hkv=1, seed=6, max_blocks=20, poison=False).upload()
    c.check(*c.run(0))


@pytest.mark.parametrize("batch, hkv, longest", [(3, 2, 900), (18, 8, 300), (30, 8, 400), (64, 8, 300), (130, 8, 300),
                                                 (170, 8, 300), (170, 8, 1100)])
def test_whole_pairs_by_groups_of_every_size(batch, hkv, longest):
    """One pair to an SM and up to ten: groups of 16, 8, 4, 2 and 1 warps, ragged lengths, empty and one-token ones."""
    lens = np.random.default_rng(batch).integers(0, longest + 1, size=batch)
    lens[:4] = [longest, 0, 1, 65][:len(lens[:4])]
    c = Case(list(lens), hkv=hkv, seed=batch, max_blocks=-(-longest // 16)).upload()
    assert c.P.puzzle_decode_attn_kernel_name(c.desc, c.view, batch) == "decode_attn_group_kernel"
    c.check(*c.run(0))
    assert int(c.status.item()) == 0


@pytest.mark.parametrize("splits", [0, -1, -2, 4])
def test_growing_logits_raise_the_reference(splits):
    """Keys that grow along the sequence: the running maximum is raised again and again, by less and by more than 2^8."""
    c = Case([1200, 640], hkv=2, seed=7, scale=1.0)
    for b in range(c.batch):
        for j in range(c.mb):
            c.k[c.table[b, j], :, 512:] = np.minimum(0x20 + 6 * j // 4, 0x48)     # the group scales, E4M3 codes upwards
    c.k_scale[:] = 0.25
    c.upload()
    # logits up to 64 * 6 * 4 * 4 * 0.25 / 8: within the bound's 200
    c.check(*c.run(splits))


def test_extreme_scales():
    """The largest group scale times the largest code (2688), and subnormal group scales: both exact in f16."""
    c = Case([200, 77], hkv=2, seed=8)
    c.k[:, :, 512:] = 0x7E
    c.k_scale[:] = 2.0 ** -9
    c.v[:, :, 512:] = 0x01
    c.v_scale[:] = 2.0 ** 9
    c.upload()
    got, lse = c.run(0)
    c.check(got, lse)


@pytest.mark.parametrize("splits", [0, -1, -2, 3])
def test_stale_and_bad_table_entries(splits):
    """Entries wholly before the window are never read; a bad entry in sight is flagged and read as zeros."""
    c = Case([700, 320], window=100, seed=9)
    c.table[0, :(700 - 100) // 16] = -1
    c.table[1, 0] = 10 ** 6
    c.upload()
    c.check(*c.run(splits))
    assert int(c.status.item()) == 0
    bad = Case([300, 320], seed=10)
    bad.table[1, 7] = 10 ** 6
    bad.upload()
    got, lse = bad.run(splits)
    assert int(bad.status.item()) == bad.P.DEV_BAD_BLOCK
    bad.check(got, lse, rows=[0])
    bad.table[1, 7] = 99
    spare = np.zeros((60, 2, 576), np.uint8)                  # the oracle sees a block of zeros there
    bad.k, bad.v = np.concatenate([bad.k, spare]), np.concatenate([bad.v, spare])
    bad.check(got, lse)


@pytest.mark.parametrize("splits", [0, -1, -2, 3])
def test_a_nan_among_the_visible_keys_is_not_hidden(splits):
    c = Case([1000, 320], hkv=2, seed=11)
    blk = c.table[0, 20]
    c.k[blk, 1, R.k_scale_at(3, 2)] = 0x7F
    c.upload()
    got, _ = c.run(splits)
    assert np.isnan(got[0, 8:]).all()
    assert not np.isnan(got[0, :8]).any() and not np.isnan(got[1]).any()
    c = Case([1000, 320], hkv=2, seed=11)
    c.v[blk, 1, R.v_scale_at(3, 2)] = 0x7F                    # channels 32 .. 47 of one token
    c.upload()
    got, _ = c.run(splits)
    assert np.isnan(got[0, 8:, 32:48]).all()
    ok = np.ones_like(got, bool)
    ok[0, 8:, 32:48] = False
    assert not np.isnan(got[ok]).any()


def test_sequences_longer_than_their_row_are_clamped_and_flagged():
    c = Case([200, 500], max_blocks=20, seed=12, poison=False).upload()
    got, lse = c.run(0)
    assert int(c.status.item()) == c.P.DEV_SEQ_TOO_LONG
    c.check(got, lse, lens=np.array([200, 320], np.int32))


def test_one_workspace_for_all_cache_types_and_batches():
    """Calls of different types, batches and splits, one after the other, on one prepared workspace."""
    import paper_2602_11937_b200 as P
    d4 = P.layer_desc(kv_dtype=P.KV_FP4_E2M1, num_q_heads=16, num_kv_heads=2)
    ws = torch.empty(max(P.puzzle_decode_attn_workspace_bytes(d4, 10, s) for s in (0, 5)), dtype=torch.uint8,
                     device="cuda").fill_(0xFF)
    P.puzzle_decode_attn_workspace_init(d4, 10, ws)
    d8 = P.layer_desc(num_q_heads=16, num_kv_heads=2)
    k8 = torch.randint(0, 100, (8, 2, 16, 64), dtype=torch.uint8, device="cuda")
    l8 = torch.tensor([120], dtype=torch.int32, device="cuda")
    v8 = P.kv_view(k8, k8, l8, max_blocks_per_seq=8)
    q8 = torch.randn(1, 16, 64, device="cuda").bfloat16()
    first = None
    for lens, splits in ((LENS, 0), ([90, 300], 5), ([2000], -1), (LENS, 5), (LENS, -2)):
        c = Case(lens, seed=len(lens) + splits).upload()
        c.check(*c.run(splits, ws))
        o8 = torch.empty_like(q8)
        P.puzzle_decode_attn(d8, v8, q8, None, o8, workspace=ws)
        torch.cuda.synchronize()
        first = o8 if first is None else first
        assert torch.allclose(o8.float(), first.float(), rtol=2.0 ** -7, atol=0)


@pytest.mark.parametrize("window", [0, 128])
def test_graph_stream_static_and_repeats(window):
    """Captured and replayed, on another stream, and through the entry point with the built-in scratch: the same values
    up to the order of float32 sums (one bf16 step)."""
    import paper_2602_11937_b200 as P
    c = Case([900, 65, 3, 0, 400], window=window, seed=13).upload()
    want, _ = c.run(0)
    out = torch.zeros(5, 16, 64, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(5, 16, device="cuda")
    q = c.d["q"][:, 0].contiguous()
    P.puzzle_decode_attn_static(c.desc, c.view, q, c.d["sinks"], out, lse)
    torch.cuda.synchronize()
    c.check(out.double().cpu().numpy(), lse.double().cpu().numpy())
    ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(c.desc, 5, 0), dtype=torch.uint8, device="cuda")
    P.puzzle_decode_attn_workspace_init(c.desc, 5, ws)
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        P.puzzle_decode_attn(c.desc, c.view, q, c.d["sinks"], out, lse, workspace=ws, stream=side)
    for _ in range(3):
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        c.check(out.double().cpu().numpy(), lse.double().cpu().numpy())


def test_partials_over_context_shards_merge_to_the_whole():
    """Blocks dealt to three shards: float32 partials without the sink, merged with it."""
    import paper_2602_11937_b200 as P
    c = Case([1000, 77, 0, 16], seed=14, poison=False).upload()
    world, hq = 3, c.hq
    buf = torch.empty(world, 4 * hq * 65, device="cuda")
    ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(c.desc, 4, 0), dtype=torch.uint8, device="cuda")
    P.puzzle_decode_attn_workspace_init(c.desc, 4, ws)
    keep = []
    for rank in range(world):
        l, _ = P.context_slice(c.d["lens"], rank, world)
        t = c.d["table"][:, rank::world].contiguous()
        keep += [t, l]
        view = P.kv_view(c.d["k"], c.d["v"], l, block_table=t, k_scale=c.d["k_scale"], v_scale=c.d["v_scale"])
        o, lse = buf[rank, :4 * hq * 64].view(4, hq, 64), buf[rank, 4 * hq * 64:].view(4, hq)
        P.puzzle_decode_attn_partial(c.desc, view, c.d["q"][:, 0].contiguous(), o, lse, workspace=ws)
    out = torch.empty(4, hq, 64, dtype=torch.bfloat16, device="cuda")
    lse_out = torch.empty(4, hq, device="cuda")
    stride = 4 * hq * 65
    P.puzzle_attn_merge_strided(buf.view(-1), buf.view(-1)[4 * hq * 64:], 64, stride, 1, stride, None, c.d["sinks"], out,
                                world, lse_out=lse_out)
    torch.cuda.synchronize()
    c.check(out.double().cpu().numpy(), lse_out.double().cpu().numpy())


def _tokens(c, ws=None):
    P = c.P
    if ws is None:
        ws = torch.empty(P.puzzle_decode_attn_tokens_workspace_bytes(c.desc, c.batch, c.n_q), dtype=torch.uint8,
                         device="cuda").fill_(0xFF)
        P.puzzle_decode_attn_tokens_workspace_init(c.desc, c.batch, c.n_q, ws)
    out = torch.full((c.batch, c.n_q, c.hq, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.batch, c.n_q, c.hq), 7.0, device="cuda")
    P.puzzle_decode_attn_tokens(c.desc, c.view, c.d["q"], c.d["sinks"], out, lse, q_lens=c.d["q_lens"], workspace=ws,
                                dev_status=c.status)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def _check_tokens(c, ws=None):
    got, lse = _tokens(c, ws)
    ql = np.full(c.batch, c.n_q) if c.q_lens is None else np.clip(c.q_lens, 0, c.n_q)
    for i in range(c.n_q):
        real = np.flatnonzero(i < ql)
        c.check(got[:, i], lse[:, i], token=i, rows=real)
        rest = np.flatnonzero(i >= ql)
        assert (got[rest, i] == 7.0).all() and (lse[rest, i] == 7.0).all()      # rows behind the last token
    assert int(c.status.item()) == 0


@pytest.mark.parametrize("n_q", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("window", [0, 1, 16, 100])
def test_several_tokens(n_q, window):
    """Every query token against the oracle's single step at its position: ragged counts, sequences shorter than their
    tokens, tokens behind the last one."""
    for q_lens in (None, [n_q, 1, 2, 0, n_q, 3, n_q, -1, 1, n_q + 4]):
        _check_tokens(Case([700, 1, 2, 16, 17, 333, 64, 65, 3, 2100], window=window, seed=n_q + window, n_q=n_q,
                           q_lens=q_lens).upload())


@pytest.mark.parametrize("batch, hkv, longest, n_q", [(3, 2, 900, 2), (18, 8, 300, 2), (16, 8, 400, 3), (16, 8, 300, 5),
                                                      (40, 8, 300, 3), (64, 8, 300, 4), (40, 8, 1100, 6), (2, 2, 9000, 3)])
def test_several_tokens_by_groups_of_every_size(batch, hkv, longest, n_q):
    """One row of two tokens to an SM and up to seven (groups of 12, 6, 4, 2, 1 warps), and the evenly cut kernel."""
    r = np.random.default_rng(batch)
    lens = r.integers(0, longest + 1, size=batch)
    lens[:4] = [longest, 1, 0, 65][:len(lens[:4])]
    _check_tokens(Case(list(lens), hkv=hkv, seed=batch, max_blocks=-(-longest // 16), n_q=n_q, poison=False,
                       q_lens=list(r.integers(0, n_q + 2, size=batch))).upload())


@pytest.mark.parametrize("hkv", [1, 3, 8])
def test_several_tokens_head_counts_without_sinks(hkv):
    _check_tokens(Case([130, 0, 257, 48], hkv=hkv, paged=hkv != 3, sinks=False, seed=hkv, n_q=3).upload())


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 63, 64, 65, 66, 127, 128, 129])
def test_several_tokens_at_tile_edges(length):
    _check_tokens(Case([length, length + 1], hkv=1, max_blocks=20, seed=length, n_q=2).upload())
    _check_tokens(Case([length, length + 1], hkv=1, max_blocks=20, seed=length, n_q=2, window=33).upload())


def test_several_tokens_on_one_workspace_and_in_a_graph():
    import paper_2602_11937_b200 as P
    d = P.layer_desc(kv_dtype=P.KV_FP4_E2M1, num_q_heads=16, num_kv_heads=2)
    ws = torch.empty(P.puzzle_decode_attn_tokens_workspace_bytes(d, 4, 5), dtype=torch.uint8, device="cuda").fill_(0xFF)
    P.puzzle_decode_attn_tokens_workspace_init(d, 4, 1, ws)
    for n_q in (5, 2, 4, 1, 5):
        c = Case([900, 65, 3, 400], seed=n_q, n_q=n_q).upload()
        _check_tokens(c, ws)
    out, lse = torch.empty_like(c.d["q"]), torch.empty(4, 5, 16, device="cuda")
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        P.puzzle_decode_attn_tokens(c.desc, c.view, c.d["q"], c.d["sinks"], out, lse, workspace=ws)
    for _ in range(2):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        for i in range(5):
            c.check(out[:, i].double().cpu().numpy(), lse[:, i].double().cpu().numpy(), token=i)


def test_single_steps_and_several_tokens_agree():
    """One decode row per query token (paging.multi_token_args) and the paired form: the same values."""
    import paper_2602_11937_b200 as P
    c = Case([700, 129, 5], seed=30, n_q=3).upload()
    lens, table = P.multi_token_args(c.d["lens"], c.d["table"], 3)
    view = P.kv_view(c.d["k"], c.d["v"], lens, block_table=table, k_scale=c.d["k_scale"], v_scale=c.d["v_scale"])
    ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(c.desc, 9, 0), dtype=torch.uint8, device="cuda")
    P.puzzle_decode_attn_workspace_init(c.desc, 9, ws)
    out = torch.empty(9, 16, 64, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(9, 16, device="cuda")
    P.puzzle_decode_attn(c.desc, view, c.d["q"].view(9, 16, 64), c.d["sinks"], out, lse, workspace=ws)
    torch.cuda.synchronize()
    for i in range(3):
        c.check(out.view(3, 3, 16, 64)[:, i].double().cpu().numpy(), lse.view(3, 3, 16)[:, i].double().cpu().numpy(), token=i)
    _check_tokens(c)


@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("lens", [[64, 129, 5], [2000, 3001, 700]])
def test_a_nan_of_one_token_stays_out_of_the_other(window, lens):
    """The newest key is not visible to the earlier token of a pair, nor the oldest one of a window to the later: a NaN there
    (K or V) is the business of the token that sees it."""
    c = Case(lens, hkv=2, seed=40, n_q=2, window=window, poison=False)
    for b, n in enumerate(lens):
        newest = c.table[b, (n - 1) // 16]
        (c.v if b != 1 else c.k)[newest, 1, (R.v_scale_at if b != 1 else R.k_scale_at)((n - 1) % 16, 2)] = 0x7F
        if window and n > window:
            t = n - 1 - window                                  # the oldest key of the earlier token
            c.v[c.table[b, t // 16], 0, R.v_scale_at(t % 16, 0)] = 0x7F
    c.upload()
    got, lse = _tokens(c)
    clean = Case(lens, hkv=2, seed=40, n_q=2, window=window, poison=False)
    for token in (0, 1):
        ref, ref_lse = clean.oracle(token)
        bad = np.isnan(got[:, token])
        for b, n in enumerate(lens):
            want = np.zeros((16, 64), bool)
            if token == 1:
                want[8:, slice(None) if b == 1 else slice(32, 48)] = True
            elif window and n > window:
                want[:8, :16] = True
            assert np.array_equal(bad[b], want), (token, b)
        clean.check(np.where(bad, ref, got[:, token]), np.where(bad.all(-1), ref_lse, lse[:, token]), token=token)
    assert int(c.status.item()) == 0


@pytest.mark.parametrize("splits", [0, -1, -2, 3])
def test_a_nan_in_a_query_head_shows_in_its_output_alone(splits):
    """All logits of the head are NaN, so that its running maximum never leaves minus infinity."""
    c = Case([1000, 1, 16], hkv=2, seed=12)
    c.q[:, 0, 11, 5] = float("nan")
    c.upload()
    got, _ = c.run(splits)
    assert np.isnan(got[:, 11]).all()
    assert not np.isnan(np.delete(got, 11, axis=1)).any()
    c = Case([1000, 5, 16], hkv=2, n_q=3, seed=12)
    c.q[:, 1, 11, 5] = float("nan")
    c.upload()
    got, _ = _tokens(c)
    assert np.isnan(got[:, 1, 11]).all()
    got[:, 1, 11] = 0
    assert not np.isnan(got).any()
