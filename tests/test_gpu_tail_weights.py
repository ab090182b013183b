"""Softmax weights far below the largest one over the E4M3 and the bf16 cache (the 4-bit one: test_gpu_fp4_weights.py): one
dominant key whose value is zero and a long context of equal keys, so that the output is the tail's share alone.

Bound on an output, relative: 2^-8 to bf16, 2^-11 for sums of up to 65536 products of one sign in the MMAs (at most 4096 in a row, off
by 2^-23 of the sum each), 2^-11 for the sum of the weights (a lane adds eight pairs of a tile one by one to the largest weight:
8192 additions at most, 2^-24 each), less than 2^-14 for logits and exponentials; a weight itself is held to 2^-16.  The same 2^-11
and 2^-14 bound the lse."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
REL = 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -11 + 2.0 ** -14 + 2.0 ** -16
LSE = 2.0 ** -11 + 2.0 ** -14
FP8, BF16 = 0, 1


def _tail(kv_dtype, octaves, n, where, hkv=1, batch=1):
    """Caches of n keys with logit 0 and value 1, but for key `where` of every sequence: `octaves` above them, value 0."""
    blocks = -(-n // 16)
    k = torch.zeros(batch, blocks, hkv, 16, 64)
    v = torch.ones_like(k)
    top = torch.tensor(6.0 if kv_dtype == FP8 else octaves * math.log(2.0) * 8.0)
    k[:, where // 16, :, where % 16, 0] = top
    v[:, where // 16, :, where % 16] = 0.0
    to = (lambda t: t.to(torch.float8_e4m3fn).view(torch.uint8)) if kv_dtype == FP8 else (lambda t: t.to(torch.bfloat16))
    scale = torch.full((hkv,), octaves * math.log(2.0) * 8.0 / 6.0)
    gap = (6.0 * float(scale[0]) if kv_dtype == FP8 else float(top.to(torch.bfloat16))) / 8.0
    keep = [to(k).flatten(0, 1).cuda(), to(v).flatten(0, 1).cuda(), scale.cuda(),
            torch.full((batch,), n, dtype=torch.int32, device="cuda")]
    tail = (n - 1) * math.exp(-gap)
    return keep, tail / (1.0 + tail), gap + math.log1p(tail)


def _view(P, kv_dtype, keep, n, hkv):
    desc = P.layer_desc(kv_dtype=kv_dtype, num_q_heads=8 * hkv, num_kv_heads=hkv)
    return desc, P.kv_view(keep[0], keep[1], keep[3], max_blocks_per_seq=-(-n // 16), k_scale=keep[2])


def _check(out, lse, want, want_lse):
    out, lse = out.double().cpu(), lse.double().cpu()
    assert ((out - want).abs() <= REL * want).all(), (float(out.min()) / want, float(out.max()) / want)
    assert ((lse - want_lse).abs() <= LSE).all()


@pytest.mark.parametrize("kv_dtype", [FP8, BF16])
@pytest.mark.parametrize("octaves", [20.0, 22.3, 24.4, 25.4, 26.0])
@pytest.mark.parametrize("where", [0, 40000])
def test_a_long_tail_far_below_one_key(octaves, where, kv_dtype):
    import paper_2602_11937_b200 as P
    n = 65536
    keep, want, want_lse = _tail(kv_dtype, octaves, n, where)
    desc, view = _view(P, kv_dtype, keep, n, 1)
    q = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    for splits in (0, 1, 4, -1, -2):
        ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(desc, 1, splits), dtype=torch.uint8, device="cuda")
        P.puzzle_decode_attn_workspace_init(desc, 1, ws)
        out, lse = torch.empty(1, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 8, device="cuda")
        P.puzzle_decode_attn(desc, view, q[:, 0].contiguous(), None, out, lse, num_splits=splits, workspace=ws)
        _check(out, lse, want, want_lse)
    if kv_dtype == FP8:
        ws = torch.empty(P.puzzle_decode_attn_tokens_workspace_bytes(desc, 1, 2), dtype=torch.uint8, device="cuda")
        P.puzzle_decode_attn_tokens_workspace_init(desc, 1, 2, ws)
        out, lse = torch.empty_like(q), torch.empty(1, 2, 8, device="cuda")
        P.puzzle_decode_attn_tokens(desc, view, q, None, out, lse, workspace=ws)
        _check(out[:, 1], lse[:, 1], want, want_lse)


@pytest.mark.parametrize("kv_dtype", [FP8, BF16])
@pytest.mark.parametrize("octaves", [20.0, 24.4, 26.0])
@pytest.mark.parametrize("n, batch", [(100, 3), (1000, 40)])
def test_a_tail_in_short_contexts(octaves, n, batch, kv_dtype):
    import paper_2602_11937_b200 as P
    keep, want, want_lse = _tail(kv_dtype, octaves, n, 3, hkv=8, batch=batch)
    desc, view = _view(P, kv_dtype, keep, n, 8)
    q = torch.zeros(batch, 64, 64, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
    P.puzzle_decode_attn_workspace_init(desc, batch, ws)
    out, lse = torch.empty_like(q), torch.empty(batch, 64, device="cuda")
    P.puzzle_decode_attn(desc, view, q, None, out, lse, workspace=ws)
    _check(out, lse, want, want_lse)
