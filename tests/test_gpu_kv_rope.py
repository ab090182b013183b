"""Append with the position rotation (all three cache types, steps and chunks), plain appends to the 4-bit cache, and the
read-back, against the plain references: cache bytes exact (also the ones that must stay as they were), rotated queries
exact bf16 bits, read-back exact."""
import numpy as np
import pytest
import torch

from helpers import bf16_bits, bits_to_bf16
import kv_reference as R

pytestmark = pytest.mark.gpu

KINDS = {"fp8": R.FP8, "bf16": R.BF16, "fp4": R.FP4}


class Setup:
    """Caches full of arbitrary bytes, a permuted table with spare blocks, ragged lengths, q/k/v cut out of one array."""

    def __init__(self, kind, seq_lens, n, hkv=2, max_blocks=9, paged=True, seed=0, rotary=64, positions=400, width=None):
        import paper_2602_11937_b200 as P
        self.P, self.kind, self.hkv, self.hq, self.n = P, kind, hkv, 8 * hkv, n
        self.lens = np.asarray(seq_lens, np.int32)
        self.batch, self.max_blocks = len(seq_lens), max_blocks
        nb = self.batch * max_blocks + (3 if paged else 0)
        r = np.random.default_rng(seed)
        self.table = r.permutation(nb)[:self.batch * max_blocks].reshape(self.batch, -1).astype(np.int32) if paged else None
        self.ref = R.Cache(kind, nb, hkv, seed + 1)
        self.k_scale, self.v_scale = ((0.003 + 0.01 * r.random(hkv)).astype(np.float32) for _ in range(2))
        self.cos_sin = P.rope_table(positions, rotary, theta=500.0).numpy()
        width = width or self.hq + 2 * hkv
        g = torch.Generator().manual_seed(seed + 2)
        self.qkv = torch.randn(self.batch, n, width, 64, generator=g).to(torch.bfloat16)
        self.rotary, self.positions = rotary, positions

    def upload(self):
        up = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
        cache = (lambda a: bits_to_bf16(a).cuda()) if self.kind == R.BF16 else up
        self.d = dict(k=cache(self.ref.k), v=cache(self.ref.v), table=up(self.table), lens=up(self.lens),
                      ks=up(self.k_scale), vs=up(self.v_scale), cs=up(self.cos_sin), qkv=self.qkv.cuda(),
                      status=torch.zeros(1, dtype=torch.int32, device="cuda"))
        self.desc = self.P.layer_desc(kv_dtype=self.kind, num_q_heads=self.hq, num_kv_heads=self.hkv)
        self.view = self.P.kv_view(self.d["k"], self.d["v"], self.d["lens"], block_table=self.d["table"],
                                   max_blocks_per_seq=self.max_blocks, k_scale=self.d["ks"], v_scale=self.d["vs"])

    def parts(self, t):
        return t[:, :, :self.hq], t[:, :, self.hq:self.hq + self.hkv], t[:, :, self.hq + self.hkv:self.hq + 2 * self.hkv]

    def cache_bits(self):
        torch.cuda.synchronize()
        if self.kind == R.BF16:
            return bf16_bits(self.d["k"]), bf16_bits(self.d["v"])
        return self.d["k"].cpu().numpy(), self.d["v"].cpu().numpy()

    def check_cache(self):
        k, v = self.cache_bits()
        assert np.array_equal(k, self.ref.k)
        assert np.array_equal(v, self.ref.v)

    def dead(self, shape):
        return torch.full(shape, 0xDEAD - 65536, dtype=torch.int16, device="cuda").view(torch.bfloat16)

    def run(self, new_lens=None, adjacent=False, offset=None, with_q=True, rotate=True):
        """Both sides; returns the device's q_out and the reference's."""
        up = lambda a: None if a is None else torch.from_numpy(np.asarray(a, np.int32)).cuda()
        q, k, v = self.parts(self.d["qkv"])
        nl, off = up(new_lens), up(offset)
        q_out = None
        if rotate:
            rope = self.P.rope_view(self.d["cs"], interleaved=adjacent, pos_offset=off)
            q_out = self.dead((self.batch, self.n, self.hq, 64)) if with_q else None
            self.P.puzzle_kv_append_rope(self.desc, self.view, rope, q if with_q else None, k, v, q_out, new_lens=nl,
                                         dev_status=self.d["status"])
        elif self.n == 1 and new_lens is None:
            self.P.puzzle_kv_append(self.desc, self.view, k[:, 0].contiguous(), v[:, 0].contiguous(),
                                    dev_status=self.d["status"])
        else:
            self.P.puzzle_kv_append_tokens(self.desc, self.view, k.contiguous(), v.contiguous(), nl,
                                           dev_status=self.d["status"])
        hq, hk, hv = (bf16_bits(x) for x in self.parts(self.qkv))
        want = R.append(self.ref, self.table, self.max_blocks, self.lens, new_lens, hq if with_q else None, hk, hv,
                        self.k_scale, self.v_scale, self.cos_sin if rotate else None, self.rotary, adjacent, offset)
        if q_out is not None:
            torch.cuda.synchronize()
            assert np.array_equal(bf16_bits(q_out), want)
        self.check_cache()
        return q_out


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 2, 5, 33, 64])
def test_append_rope_bytes(kind, n):
    """Every type, steps and chunks that start at even and odd slots, cross blocks, are cut short, or are skipped."""
    s = Setup(KINDS[kind], [144, n, 0, 7, 66, 97], n, seed=n)
    s.upload()
    s.run()
    s.run(new_lens=[n, 0, 3, min(n, 4), -1, n + 5])
    assert int(s.d["status"].item()) == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rotary, adjacent", [(16, False), (32, False), (48, False), (16, True), (48, True), (64, True)])
@pytest.mark.parametrize("n", [1, 6])
def test_rotation_forms(kind, rotary, adjacent, n):
    s = Setup(KINDS[kind], [100, 6, 41], n, seed=rotary, rotary=rotary)
    s.upload()
    s.run(adjacent=adjacent)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hkv", [1, 3, 8, 9])
def test_head_counts_contiguous_cache_and_no_queries(kind, hkv):
    for n in (1, 7):
        s = Setup(KINDS[kind], [50, 20], n, hkv=hkv, paged=False, seed=hkv, width=10 * hkv + 2)
        s.upload()
        s.run()
        s.run(with_q=False)


@pytest.mark.parametrize("n", [1, 2, 19, 40])
def test_plain_appends_to_the_4bit_cache(n):
    s = Setup(R.FP4, [144, n, 0, 7, 66, 97], n, seed=n + 7)
    s.upload()
    s.run(rotate=False)
    s.run(rotate=False, new_lens=[n, 0, 3, min(n, 4), -1, n + 5])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 9])
def test_offsets_and_positions_outside_the_table(kind, n):
    """offset moves a token's position, not its place; positions the table lacks are flagged and skipped."""
    s = Setup(KINDS[kind], [100, 60, 30, 20], n, seed=5)
    s.upload()
    s.run(offset=[250, 0, -3, 17])
    assert int(s.d["status"].item()) == 0
    s.run(offset=[303, 2 ** 31 - 40, -25, 0])       # past the end from the fifth token on, far past it, before the start
    assert int(s.d["status"].item()) == s.P.DEV_BAD_POSITION


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 20])
def test_bad_blocks_and_rows_that_are_too_long(kind, n):
    s = Setup(KINDS[kind], [100, 145, 60], n, seed=8)
    s.table[0, 6] = 10 ** 6
    s.table[2, 3] = -1
    s.upload()
    s.run()
    assert int(s.d["status"].item()) == s.P.DEV_BAD_BLOCK | s.P.DEV_SEQ_TOO_LONG


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 6])
def test_unusual_values(kind, n):
    """Zeros of both signs, infinities, NaN, the largest bf16, subnormals, and groups of one tiny channel."""
    s = Setup(KINDS[kind], [40, 17], n, seed=9)
    v = s.qkv.view(torch.int16)
    v[0, 0, :, 3], v[0, 0, :, 20], v[0, 0, :, 50] = 0x7F80, 0x7FC0, -0x80          # +inf, NaN, -inf
    v[0, -1, 1] = 0x7F7F
    v[1, 0, :] = -0x8000                                                             # -0
    v[1, 0, :, 33] = 0x0001
    v[1, -1, :, 1::2] = 0x0100                                                       # 2^-125
    s.upload()
    s.run()


@pytest.mark.parametrize("scale", [1.0, 2.0 ** -7, 0.1, 3.0, 2.0 ** 70, 1.5 * 2.0 ** -80])
@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_scales_of_every_kind(kind, scale):
    """Powers of two, others, and scales beyond the range of the corrected reciprocal."""
    s = Setup(KINDS[kind], [90, 31, 64], 31, seed=10)
    s.k_scale[:] = scale
    s.v_scale[:] = np.float32(scale) * np.float32(1.0 + 2.0 ** -23)
    s.upload()
    s.run()


def test_quotients_round_as_a_division_does():
    """Every bf16 significand over scales with awkward significands, values next to and on code borders: the corrected
    reciprocal gives the byte that the IEEE quotient gives."""
    import paper_2602_11937_b200 as P
    r = np.random.default_rng(4)
    n = 512
    for seed in range(6):
        s = Setup(R.FP8, [n, n], n, max_blocks=n // 16, seed=seed, positions=n)
        s.k_scale[:] = np.float32(1.0) + r.integers(1, 1 << 23, 2).astype(np.float32) * np.float32(2.0 ** -23)
        s.v_scale[:] = [np.float32(2.0) - np.float32(2.0 ** -23), np.float32(1.0 + 2.0 ** -23)]
        s.upload()
        s.run(with_q=False)


@pytest.mark.parametrize("n", [1, 12])
def test_in_place_queries_and_a_graph(n):
    """q_out == q, captured and replayed: the second replay turns the queries a second time, the cache's bytes stay."""
    s = Setup(R.FP4, [90, 44], n, seed=12)
    s.upload()
    P = s.P
    q, k, v = (x.contiguous() for x in s.parts(s.d["qkv"]))
    rope = P.rope_view(s.d["cs"])
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        P.puzzle_kv_append_rope(s.desc, s.view, rope, q, k, v, q, dev_status=s.d["status"])
    hq, hk, hv = (bf16_bits(x) for x in s.parts(s.qkv))
    for _ in range(2):
        g.replay()
        hq = R.append(s.ref, s.table, s.max_blocks, s.lens, None, hq, hk, hv, s.k_scale, s.v_scale, s.cos_sin)
        torch.cuda.synchronize()
        assert np.array_equal(bf16_bits(q), hq)
        s.check_cache()


def test_another_stream_and_no_scales():
    s = Setup(R.FP4, [90, 44], 5, seed=13)
    s.k_scale[:] = s.v_scale[:] = 1.0
    s.upload()
    s.view = s.P.kv_view(s.d["k"], s.d["v"], s.d["lens"], block_table=s.d["table"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    side.synchronize()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 3, 70])
@pytest.mark.parametrize("hkv", [1, 8, 9])
def test_read_back(kind, n, hkv):
    """Every byte pattern reads as its value times the scale, rounded to float32 and then to bf16; rows that are not
    asked for stay as they were."""
    s = Setup(KINDS[kind], [144, 2, 0, 37, 145], n, hkv=hkv, seed=n, max_blocks=9)
    s.table[3, 1] = 10 ** 6
    s.upload()
    for lens in (None, [n, 1, n, 0, n]):
        want = {w: np.full((s.batch, n, hkv, 64), 0xDEAD, np.uint16) for w in "kv"}
        for b in range(s.batch):
            count = n if lens is None else lens[b]
            if s.lens[b] > 144:
                continue
            for i in range(count):
                pos = s.lens[b] - count + i
                if pos < 0:
                    continue
                blk = s.table[b, pos // 16]
                for h in range(hkv):
                    for w in "kv":
                        if blk >= s.ref.k.shape[0]:
                            want[w][b, i, h] = 0
                        elif s.kind == R.BF16:
                            want[w][b, i, h] = (s.ref.v if w == "v" else s.ref.k)[blk, h, pos % 16]
                        else:
                            scale = (s.v_scale if w == "v" else s.k_scale)[h]
                            x = s.ref.get(blk, pos % 16, h, w == "v").astype(np.float32)
                            want[w][b, i, h] = R.round_bf16(x * scale)
        out = {w: s.dead((s.batch, n, hkv, 64)) for w in "kv"}
        s.d["status"].zero_()
        s.P.puzzle_kv_read_tokens(s.desc, s.view, out["k"], out["v"],
                                  None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                  dev_status=s.d["status"])
        torch.cuda.synchronize()
        assert int(s.d["status"].item()) & s.P.DEV_SEQ_TOO_LONG
        for w in "kv":
            got = bf16_bits(out[w])
            nan = np.isnan(bits_to_bf16(want[w]).float().numpy()) & (want[w] != 0xDEAD)
            if s.kind != R.BF16:                       # the sign of a NaN product is not defined
                assert np.array_equal(nan, np.isnan(bits_to_bf16(got).float().numpy()) & (got != 0xDEAD))
                got, ref = np.where(nan, 0, got), np.where(nan, 0, want[w])
            else:
                ref = want[w]
            assert np.array_equal(got, ref)


@pytest.mark.parametrize("kind", KINDS)
def test_append_then_read(kind):
    """What an append wrote is what the read-back gives: x to within half a step of its code."""
    import paper_2602_11937_b200 as P
    s = Setup(KINDS[kind], [130, 77], 50, seed=21)
    s.upload()
    q_out = s.run()
    k, v = (torch.empty(2, 50, s.hkv, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    P.puzzle_kv_read_tokens(s.desc, s.view, k, v)
    x = s.parts(s.qkv)[2].double()
    err = (v.cpu().double() - x).abs()
    scale = torch.from_numpy(s.v_scale).double()[:, None]
    if kind == "bf16":
        bound = torch.zeros_like(x)
    elif kind == "fp8":
        # half a step of E4M3 relative to the value, half the smallest step near zero; bf16 on top.  The largest code is
        # 448 and the smallest scale here 0.003, so |x| > 1.344 may saturate: the code then stands for 448 scale, and
        # the error is |x| - 448 scale exactly (the code nearest to x / scale is the largest one)
        bound = x.abs() * 2.0 ** -4 + scale * 2.0 ** -10 + (x.abs() - 448 * scale).clamp(min=0)
    else:
        # group scale t: off by half a step of E4M3 (2^-4), so codes reach 6 (1 + 2^-4) and saturate by 6 * 2^-4 t at
        # most; otherwise half an E2M1 step, 1 t at most (between 4 and 6); t <= (1 + 2^-4) amax / 6
        t = (1 + 2.0 ** -4) * x.unflatten(-1, (4, 16)).abs().amax(-1, keepdim=True) / 6
        bound = (t.expand(-1, -1, -1, -1, 16).flatten(-2)) * 1.0 + scale * 2.0 ** -9
    bound = bound + (x.abs() + bound) * 2.0 ** -8 * (kind != "bf16")
    assert bool((err <= bound).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("batch, n", [(3, 1), (1, 5), (1, 1)])
def test_the_stride_of_a_dimension_of_one_means_nothing(kind, batch, n):
    s = Setup(KINDS[kind], [70, 5, 33][:batch], n, seed=21)
    s.upload()
    parts = s.parts

    def odd(t):
        return [x.as_strided(x.shape, (x.stride(0) if batch > 1 else 3, x.stride(1) if n > 1 else 7, 64, 1),
                             x.storage_offset()) for x in parts(t)]
    s.parts = odd
    s.run()
