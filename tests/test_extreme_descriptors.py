"""Sizes at the ends of what the descriptors can say: windows as long as an int32 goes, table rows whose tokens an int32 cannot
count, more KV heads than a grid dimension holds."""
import ctypes

import pytest
import torch

OK, SHAPE, UNSUPPORTED = 0, 2, 3
WIDEST = [2 ** 31 - 1, 2 ** 31 - 63, 2 ** 31 - 32, 2 ** 30]


def _view(blocks=1 << 16, row=1 << 12):
    from paper_2602_11937_b200 import binding as B
    kv = B.KVView()
    kv.k_cache, kv.v_cache, kv.seq_lens, kv.block_table = 0x1000, 0x2000, 0x3000, 0x4000
    kv.num_blocks, kv.max_blocks_per_seq = blocks, row
    return kv


@pytest.mark.parametrize("kv_dtype", [0, 1, 2])
@pytest.mark.parametrize("batch", [1, 16, 300])
def test_a_window_beyond_every_context_is_no_window(kv_dtype, batch):
    """The kernel is chosen by the tiles that a sequence can have: as for a layer without a window."""
    import paper_2602_11937_b200 as P
    want = P.puzzle_decode_attn_kernel_name(P.layer_desc(kv_dtype=kv_dtype), _view(), batch)
    assert want != "decode_attn_small_kernel"
    for window in WIDEST:
        assert P.puzzle_decode_attn_kernel_name(P.layer_desc(window=window, kv_dtype=kv_dtype), _view(), batch) == want


@pytest.mark.gpu
@pytest.mark.parametrize("kv_dtype", [0, 1, 2])
def test_the_widest_windows_see_every_key(kv_dtype):
    import paper_2602_11937_b200 as P
    n, batch = 5000, 3
    blocks = -(-n // 16)
    g = torch.Generator().manual_seed(kv_dtype)
    k, v = (torch.randn(batch, n, 8, 64, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    lens = torch.tensor([n, 700, 1], dtype=torch.int32, device="cuda")
    shape = {0: (16, 64), 1: (16, 64), 2: (576,)}[kv_dtype]
    caches = [torch.zeros(batch * blocks, 8, *shape, dtype=torch.bfloat16 if kv_dtype == 1 else torch.uint8, device="cuda")
              for _ in range(2)]
    view = P.kv_view(*caches, lens, max_blocks_per_seq=blocks)
    P.puzzle_kv_append_tokens(P.layer_desc(kv_dtype=kv_dtype), view, k, v, new_lens=lens)
    q = torch.randn(batch, 2, 64, 64, generator=g).to(torch.bfloat16).cuda()
    q1 = q[:, 0].contiguous()
    want, lse = None, None
    for window in [0] + WIDEST:
        d = P.layer_desc(window=window, kv_dtype=kv_dtype)
        ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(d, batch), dtype=torch.uint8, device="cuda")
        P.puzzle_decode_attn_workspace_init(d, batch, ws)
        got, got_lse = [torch.empty_like(q1)], [torch.empty(batch, 64, device="cuda")]
        P.puzzle_decode_attn(d, view, q1, None, got[0], got_lse[0], workspace=ws)
        if kv_dtype != 1:
            wt = torch.empty(P.puzzle_decode_attn_tokens_workspace_bytes(d, batch, 2), dtype=torch.uint8, device="cuda")
            P.puzzle_decode_attn_tokens_workspace_init(d, batch, 2, wt)
            got.append(torch.empty_like(q))
            got_lse.append(torch.empty(batch, 2, 64, device="cuda"))
            P.puzzle_decode_attn_tokens(d, view, q, None, got[1], got_lse[1], workspace=wt)
        torch.cuda.synchronize()
        if want is None:
            want, lse = got, got_lse
            continue
        # the same kernel and the same weights, float32 sums in another order at most: one bf16 step, and for outputs near
        # zero 5000 * 2^-24 of the weighted mean of |v| (below 1)
        for a, b, c, e in zip(got, want, got_lse, lse):
            assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -7, atol=5000 * 2.0 ** -24)
            finite = torch.isfinite(e)                       # the earlier token of the one-token sequence sees no key
            assert torch.equal(torch.isfinite(c), finite) and torch.allclose(c[finite], e[finite], rtol=0, atol=1e-5)


@pytest.mark.parametrize("kv_dtype", [0, 1, 2])
def test_table_rows_whose_tokens_an_int32_cannot_count(kv_dtype):
    """From 2^27 blocks of 16 tokens on every length counted as too long for its row."""
    from paper_2602_11937_b200 import binding as B
    lib, d = B._load(), B.layer_desc(kv_dtype=kv_dtype)
    ref = ctypes.byref
    for row in ((1 << 26) + 1, 1 << 27, 2 ** 31 - 1):
        kv = _view(row=row)
        assert lib.puzzle_decode_attn(ref(d), ref(kv), 0x5000, None, 0x8000, None, 4, 0, 0x10000, 1 << 30, None, None) == UNSUPPORTED
        assert lib.puzzle_decode_attn_tokens(ref(d), ref(kv), 0x5000, None, None, 0x8000, None, 4, 2, 0x10000, 1 << 30, None,
                                             None) == UNSUPPORTED
        assert lib.puzzle_kv_append(ref(d), ref(kv), 0x6000, 0x7000, 4, None, None) == UNSUPPORTED
        assert lib.puzzle_kv_append_tokens(ref(d), ref(kv), 0x6000, 0x7000, None, 4, 2, None, None) == UNSUPPORTED
        assert lib.puzzle_kv_read_tokens(ref(d), ref(kv), 0x9000, 0xA000, None, 4, 2, None, None) == UNSUPPORTED
        rope, qkv = B.Rope(0x4000, 1024, 64, 0, None), B.QKV(None, 0x6000, 0x7000, 0, 0, 512, 512, 512, 512)
        assert lib.puzzle_kv_append_rope(ref(d), ref(kv), ref(rope), ref(qkv), None, None, 4, 1, None, None) == UNSUPPORTED
    kv = _view(row=1 << 26)
    assert lib.puzzle_decode_attn(ref(d), ref(kv), 0x5000, None, 0x8000, None, 4, 0, None, 0, None, None) == 4   # the workspace


def test_a_step_from_host_memory_refuses_before_it_copies():
    """More KV heads than an append to a 4-bit cache takes: found before the first copy is enqueued (here there is no device to
    copy to, so a copy would show as a CUDA error)."""
    from paper_2602_11937_b200 import binding as B
    lib, d = B._load(), B.layer_desc(kv_dtype=B.KV_FP4_E2M1, num_q_heads=8 * 4097, num_kv_heads=4097)
    kv = _view(blocks=1 << 10)
    staging = lib.puzzle_decode_step_host_staging_bytes(ctypes.byref(d), 2)
    ws = lib.puzzle_decode_attn_workspace_bytes(ctypes.byref(d), 2, 0)
    assert lib.puzzle_decode_step_host(ctypes.byref(d), ctypes.byref(kv), 0x100, 0x200, 0x300, None, 0x400, 2, 0, 0x10000, staging,
                                       0x10000, ws, None, None) == UNSUPPORTED
