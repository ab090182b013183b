"""A descriptor holds pointers; what the tensors behind them hold is noted beside it and checked before a launch: as many
sequences, scales and cache bytes as the call reads.  The checks come before any tensor is looked at, so they run without a GPU."""
import pytest
import torch

FULL = 4 * 8                       # (block, KV head) pairs of the cache below


def _view(dtype_bytes=1024, sequences=2, scales=8, blocks=4):
    from paper_2602_11937_b200 import binding as B
    v = B.KVView()
    v.num_blocks, v.max_blocks_per_seq = blocks, 2
    v._held = (0, sequences, scales, FULL * dtype_bytes)
    return v


def _calls(P, batch=2):
    """Every native call, as a function of descriptor and view; host tensors, so that what passes is refused as such."""
    z = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16)
    ws = torch.zeros(4, dtype=torch.uint8)
    return {
        "append": lambda d, v: P.puzzle_kv_append(d, v, z(batch, 8, 64), z(batch, 8, 64)),
        "append_tokens": lambda d, v: P.puzzle_kv_append_tokens(d, v, z(batch, 3, 8, 64), z(batch, 3, 8, 64)),
        "append_rope": lambda d, v: P.puzzle_kv_append_rope(d, v, P.Rope(), None, z(batch, 8, 64), z(batch, 8, 64)),
        "read": lambda d, v: P.puzzle_kv_read_tokens(d, v, z(batch, 3, 8, 64), z(batch, 3, 8, 64)),
        "attn": lambda d, v: P.puzzle_decode_attn(d, v, z(batch, 64, 64), None, z(batch, 64, 64), workspace=ws),
        "tcgen05": lambda d, v: P.puzzle_decode_attn_tcgen05(d, v, z(batch, 64, 64), None, z(batch, 64, 64), workspace=ws),
        "tokens": lambda d, v: P.puzzle_decode_attn_tokens(d, v, z(batch, 3, 64, 64), None, z(batch, 3, 64, 64), workspace=ws),
    }


NAMES = ["append", "append_tokens", "append_rope", "read", "attn", "tcgen05", "tokens"]


@pytest.mark.parametrize("name", NAMES)
def test_more_sequences_than_the_view_has(name):
    import paper_2602_11937_b200 as P
    f = _calls(P, batch=3)[name]
    with pytest.raises(ValueError, match="the cache view has 2 sequences, the call needs 3"):
        f(P.layer_desc(), _view())


@pytest.mark.parametrize("name", NAMES)
def test_a_cache_of_another_type(name):
    """A 4-bit cache under an E4M3 descriptor would be read past its end."""
    import paper_2602_11937_b200 as P
    f = _calls(P)[name]
    for dtype, need, has in ((P.KV_FP8_E4M3, 1024, 576), (P.KV_BF16, 2048, 1024), (P.KV_FP4_E2M1, 576, 575)):
        if dtype != P.KV_FP8_E4M3 and (name == "tcgen05" or (name, dtype) == ("tokens", P.KV_BF16)):
            continue                # the library refuses the type itself, with a code
        with pytest.raises(ValueError, match="the cache has %d bytes, the descriptor's 4 blocks need %d" % (FULL * has, FULL * need)):
            f(P.layer_desc(kv_dtype=dtype), _view(has))
    with pytest.raises(ValueError, match="the descriptor's 5 blocks need"):
        f(P.layer_desc(), _view(blocks=5))


@pytest.mark.parametrize("name", NAMES)
def test_fewer_scales_than_heads(name):
    import paper_2602_11937_b200 as P
    f = _calls(P)[name]
    with pytest.raises(ValueError, match="the cache view has 7 scales, the call needs 8"):
        f(P.layer_desc(), _view(scales=7))


def test_fewer_offsets_than_sequences():
    import paper_2602_11937_b200 as P
    k, r = torch.zeros(2, 8, 64, dtype=torch.bfloat16), P.Rope()
    r._held = (0, 1)
    with pytest.raises(ValueError, match="the rotation has offsets for 1 sequences, the call needs 2"):
        P.puzzle_kv_append_rope(P.layer_desc(), P.KVView(), r, None, k, k)


@pytest.mark.gpu
def test_what_a_view_notes():
    import paper_2602_11937_b200 as P
    k = torch.zeros(4, 8, 576, dtype=torch.uint8, device="cuda")
    lens = torch.ones(2, dtype=torch.int32, device="cuda")
    table = torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    scale = torch.ones(8, device="cuda")
    view = P.kv_view(k, torch.zeros(5, 8, 576, dtype=torch.uint8, device="cuda"), lens, table, k_scale=scale, v_scale=scale[:7])
    assert view._held == (0, 2, 7, 4 * 8 * 576)
    assert P.kv_view(k, k, table[:, 0].contiguous(), table[:1], k_scale=scale)._held == (0, 1, 8, 4 * 8 * 576)
    assert P.rope_view(P.rope_table(8).cuda(), pos_offset=lens)._held == (0, 2)
    q, x = torch.zeros(2, 64, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(P.puzzle_decode_attn_workspace_bytes(P.layer_desc(), 2), dtype=torch.uint8, device="cuda")
    before = P.puzzle_launch_count()
    view = P.kv_view(k, k.clone(), lens, max_blocks_per_seq=2)
    with pytest.raises(ValueError, match="the cache has 18432 bytes, the descriptor's 4 blocks need 32768"):
        P.puzzle_decode_attn(P.layer_desc(), view, q, None, torch.empty_like(q), workspace=ws)
    one = P.kv_view(k, k.clone(), lens[:1], max_blocks_per_seq=2)
    with pytest.raises(ValueError, match="the cache view has 1 sequences, the call needs 2"):
        P.puzzle_kv_append(P.layer_desc(kv_dtype=P.KV_FP4_E2M1), one, x, x)
    r = P.rope_view(P.rope_table(8).cuda(), pos_offset=lens[:1])
    with pytest.raises(ValueError, match="the rotation has offsets for 1 sequences"):
        P.puzzle_kv_append_rope(P.layer_desc(kv_dtype=P.KV_FP4_E2M1), view, r, None, x, x)
    assert P.puzzle_launch_count() == before


def test_a_field_set_by_hand_ends_what_was_noted():
    """The pointers may lead to other tensors then; nothing is known of those, and the call is not held to the old ones."""
    import paper_2602_11937_b200 as P
    for name in ("seq_lens", "block_table", "k_cache", "num_blocks", "k_scale"):
        v = _view()
        setattr(v, name, 64)
        assert v._held is None
        with pytest.raises(ValueError, match="k_new must be a CUDA tensor"):
            _calls(P, batch=3)["append"](P.layer_desc(), v)
    r = P.Rope()
    r._held = (0, 1)
    r.pos_offset = 64
    assert r._held is None
