"""Softmax weights far below the largest one, over the 4-bit cache: one dominant key whose value is zero and a long context of
equal keys, so that the output is the tail's share alone.

Bound on an output, relative, from the roundings: 2^-8 to bf16, 2^-11 of every weight to f16, 2^-11 for sums of up to 65536
products of one sign (at most 4096 MMAs in a row, off by 2^-23 of the sum each), and less than 2^-14 for the logits (one
product, times the logit scale, both off by 2^-24 of at most 120 octaves) and the exponentials.  Weights 2^-26 below the
largest one still have all their bits, so nothing absolute is added.  lse: at most 1024 tiles' sums are added one by one to
the largest weight, off by 2^-24 of it each, 2^-14 = 6.1e-5 together, and what the logits give."""
import math

import numpy as np
import pytest
import torch

import kv_reference as R

pytestmark = pytest.mark.gpu
REL = 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -11 + 2.0 ** -14


def _tail(octaves, n, where, hkv=1, batch=1):
    """Caches of n keys with logit 0 and value 1, but for key `where` of every sequence: `octaves` above them, value 0."""
    blocks = -(-n // 16)
    k = np.zeros((batch * blocks, hkv, 576), np.uint8)
    v = np.zeros_like(k)
    k[:, :, 512:] = v[:, :, 512:] = 0x38                           # group scales of 1
    v[:, :, :512] = 0x22                                           # codes of 1.0
    for b in range(batch):
        blk, t = b * blocks + where // 16, where % 16
        k[blk, :, 32 * t] = 0x07                                   # channel 0: 6.0
        for d in range(64):
            at = 256 * (d // 32) + 32 * (t // 2) + d % 32
            v[blk, :, at] &= 0x0F if t % 2 else 0xF0
    k_scale = np.full(hkv, octaves * math.log(2.0) * 8.0 / 6.0, np.float32)
    gap = 6.0 * float(k_scale[0]) / 8.0                            # q is 1 in channel 0, the logit scale 1/8
    tail = (n - 1) * math.exp(-gap)
    return k, v, k_scale, tail / (1.0 + tail), gap + math.log1p(tail)


def _device(P, n, k, v, k_scale, batch, hkv):
    up = lambda a: torch.from_numpy(a).cuda()
    keep = (up(k), up(v), up(k_scale), torch.full((batch,), n, dtype=torch.int32, device="cuda"))
    desc = P.layer_desc(kv_dtype=P.KV_FP4_E2M1, num_q_heads=8 * hkv, num_kv_heads=hkv)
    view = P.kv_view(keep[0], keep[1], keep[3], max_blocks_per_seq=-(-n // 16), k_scale=keep[2])
    return keep, desc, view


def _check(out, lse, want, want_lse):
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert (np.abs(out - want) <= REL * want).all(), (out.min() / want, out.max() / want)
    assert (np.abs(lse - want_lse) <= 1e-4).all()


@pytest.mark.parametrize("octaves", [20.0, 22.3, 24.4, 25.4, 26.0])
@pytest.mark.parametrize("where", [0, 40000])
def test_a_long_tail_far_below_one_key(octaves, where):
    import paper_2602_11937_b200 as P
    n = 65536
    k, v, k_scale, want, want_lse = _tail(octaves, n, where)
    keep, desc, view = _device(P, n, k, v, k_scale, 1, 1)
    q = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    for splits in (0, 1, 4, -1, -2):
        ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(desc, 1, splits), dtype=torch.uint8, device="cuda")
        P.puzzle_decode_attn_workspace_init(desc, 1, ws)
        out, lse = torch.empty(1, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 8, device="cuda")
        P.puzzle_decode_attn(desc, view, q[:, 0].contiguous(), None, out, lse, num_splits=splits, workspace=ws)
        _check(out, lse, want, want_lse)
    ws = torch.empty(P.puzzle_decode_attn_tokens_workspace_bytes(desc, 1, 2), dtype=torch.uint8, device="cuda")
    P.puzzle_decode_attn_tokens_workspace_init(desc, 1, 2, ws)
    out, lse = torch.empty_like(q), torch.empty(1, 2, 8, device="cuda")
    P.puzzle_decode_attn_tokens(desc, view, q, None, out, lse, workspace=ws)
    _check(out[:, 1], lse[:, 1], want, want_lse)
    tail = want / (1.0 - want) * (n - 2) / (n - 1)                 # the earlier token sees one key less
    _check(out[:, 0], lse[:, 0], tail / (1.0 + tail), want_lse - math.log1p(want / (1.0 - want)) + math.log1p(tail))


@pytest.mark.parametrize("octaves", [20.0, 24.4, 26.0])
@pytest.mark.parametrize("n, batch", [(200, 3), (1000, 40)])
def test_a_tail_in_short_contexts(octaves, n, batch):
    """The narrow-window kernel, and groups that take whole pairs."""
    import paper_2602_11937_b200 as P
    k, v, k_scale, want, want_lse = _tail(octaves, n, 3, hkv=8, batch=batch)
    keep, desc, view = _device(P, n, k, v, k_scale, batch, 8)
    q = torch.zeros(batch, 64, 64, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
    P.puzzle_decode_attn_workspace_init(desc, batch, ws)
    out, lse = torch.empty_like(q), torch.empty(batch, 64, device="cuda")
    P.puzzle_decode_attn(desc, view, q, None, out, lse, workspace=ws)
    _check(out, lse, want, want_lse)


@pytest.mark.parametrize("step", [0.9, 3.1, 14.9, 16.0])
def test_a_reference_that_is_raised_by_little_and_by_much(step):
    """One key per tile that is `step` octaves above the one before: weights between 2^12 and 2^15 of the reference, and
    beyond.  Every value is 1 but the last key's, which is 0."""
    import paper_2602_11937_b200 as P
    tiles = int(min(20, 120 // step)) & ~1 or 2
    n = 64 * tiles
    k, v, _, _, _ = _tail(1.0, n, n - 1)
    scales = np.array([1.0 + i / 8 for i in range(8)])
    for i in range(tiles):                                          # logits 0 .. in steps, as E2M1 x E4M3 products
        k[4 * i + 3, :, 32 * 15] = 0x07 if i == tiles - 1 else 0x02
        top = (i + 1) * step / (6.0 if i == tiles - 1 else 1.0)
        e = max(math.floor(math.log2(top)), -6)
        m = int(np.abs(scales - top / 2.0 ** e).argmin())
        k[4 * i + 3, :, R.k_scale_at(15, 0)] = ((e + 7) << 3) | m
    unit = math.log(2.0) * 8.0
    k_scale = np.full(1, unit, np.float32)
    value = R.E4M3[k[:, 0, 512:]].astype(np.float64)
    gap = np.zeros(n)
    for i in range(tiles):
        code = 6.0 if i == tiles - 1 else 1.0
        gap[64 * i + 63] = code * value[4 * i + 3, R.k_scale_at(15, 0) - 512] * float(k_scale[0]) / 8.0
    w = np.exp(gap - gap.max())
    want, want_lse = w[:-1].sum() / w.sum(), gap.max() + math.log(w.sum())
    keep, desc, view = _device(P, n, k, v, k_scale, 1, 1)
    q = torch.zeros(1, 8, 64, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    for splits in (0, 1, -1):
        ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(desc, 1, splits), dtype=torch.uint8, device="cuda")
        P.puzzle_decode_attn_workspace_init(desc, 1, ws)
        out, lse = torch.empty_like(q), torch.empty(1, 8, device="cuda")
        P.puzzle_decode_attn(desc, view, q, None, out, lse, num_splits=splits, workspace=ws)
        _check(out, lse, want, want_lse)
