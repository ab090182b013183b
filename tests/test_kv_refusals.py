"""Argument errors of the append with rotation, the read-back and the 4-bit cache: found on the host before anything is
launched, so they are tested without a GPU (the pointers are never followed)."""
import ctypes

import pytest
import torch

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4


def _args(kv_dtype=2, **over):
    from paper_2602_11937_b200 import binding as B
    desc = B.layer_desc(kv_dtype=kv_dtype, **{k: over.pop(k) for k in ("window", "head_dim", "num_q_heads", "block_size")
                                              if k in over})
    kv = B.KVView()
    kv.k_cache, kv.v_cache, kv.seq_lens = 0x1000, 0x2000, 0x3000
    kv.num_blocks, kv.max_blocks_per_seq = 64, 16
    rope = B.Rope(0x4000, 1024, 64, 0, None)
    qkv = B.QKV(0x5000, 0x6000, 0x7000, 4096, 4096, 512, 512, 512, 512)
    d = dict(desc=desc, kv=kv, rope=rope, qkv=qkv, q_out=0x8000, new_lens=None, batch=4, n_new=1)
    for k, v in over.items():
        where, _, field = k.partition("__")
        if field:
            setattr(d[where], field, v)
        else:
            d[k] = v
    return B._load(), d


def _append(**over):
    lib, d = _args(**over)
    ref = lambda x: ctypes.byref(x) if x is not None else None
    return lib.puzzle_kv_append_rope(ref(d["desc"]), ref(d["kv"]), ref(d["rope"]), ref(d["qkv"]), d["q_out"], d["new_lens"],
                                     d["batch"], d["n_new"], None, None)


@pytest.mark.parametrize("over, want", [
    (dict(desc=None), NULL), (dict(kv=None), NULL), (dict(rope=None), NULL), (dict(qkv=None), NULL),
    (dict(rope__cos_sin=None), NULL), (dict(qkv__k=None), NULL), (dict(qkv__v=None), NULL), (dict(q_out=None), NULL),
    (dict(kv__seq_lens=None), NULL), (dict(kv__k_cache=0x1004), SHAPE), (dict(kv_dtype=3), SHAPE),
    (dict(head_dim=128), UNSUPPORTED), (dict(num_q_heads=32), UNSUPPORTED), (dict(block_size=32), UNSUPPORTED),
    (dict(batch=0), SHAPE), (dict(batch=5000), UNSUPPORTED), (dict(n_new=0), SHAPE), (dict(n_new=(1 << 20) + 1), SHAPE),
    (dict(rope__num_positions=0), SHAPE), (dict(rope__rotary_dim=0), SHAPE), (dict(rope__rotary_dim=80), SHAPE),
    (dict(rope__rotary_dim=24), UNSUPPORTED), (dict(rope__cos_sin=0x4008), SHAPE), (dict(qkv__q=0x5008), SHAPE),
    (dict(qkv__k=0x6008), SHAPE), (dict(qkv__v=0x7002), SHAPE), (dict(q_out=0x8008), SHAPE),
    (dict(qkv__k_token_stride=-8, n_new=2), SHAPE), (dict(qkv__v_seq_stride=12), SHAPE),
    (dict(qkv__q_token_stride=4100, n_new=2), SHAPE), (dict(qkv__q_seq_stride=4100), SHAPE),
    # in place on a slice of a wider array: a row would land on another one that has not been read
    (dict(q_out=0x5000, qkv__q_seq_stride=5120), SHAPE), (dict(q_out=0x5000, n_new=2, qkv__q_token_stride=5120), SHAPE),
])
def test_append_rope_refusals(over, want):
    assert _append(**over) == want


@pytest.mark.parametrize("over, want", [
    (dict(desc=None), NULL), (dict(kv=None), NULL), (dict(k_out=None), NULL), (dict(v_out=None), NULL),
    (dict(n_new=0), SHAPE), (dict(n_new=(1 << 24) + 1), SHAPE), (dict(k_out=0x9008), SHAPE), (dict(v_out=0x9002), SHAPE),
    (dict(batch=0), SHAPE), (dict(kv__num_blocks=63), SHAPE), (dict(head_dim=128), UNSUPPORTED),
])
def test_read_tokens_refusals(over, want):
    out = {"k_out": 0x9000, "v_out": 0xA000}
    out.update({k: over.pop(k) for k in list(over) if k in out})
    lib, d = _args(**over)
    ref = lambda x: ctypes.byref(x) if x is not None else None
    assert lib.puzzle_kv_read_tokens(ref(d["desc"]), ref(d["kv"]), out["k_out"], out["v_out"], None, d["batch"], d["n_new"],
                                     None, None) == want


def test_fp4_plain_append_needs_aligned_rows():
    """The 4-bit append reads rows 16 bytes at a time."""
    lib, d = _args()
    call = lambda k, v: lib.puzzle_kv_append(ctypes.byref(d["desc"]), ctypes.byref(d["kv"]), k, v, 4, None, None)
    assert call(0x6004, 0x7000) == SHAPE and call(0x6000, 0x7008) == SHAPE and call(None, 0x7000) == NULL


def test_tcgen05_kernel_refuses_a_4bit_cache():
    lib, d = _args()
    assert lib.puzzle_decode_attn_tcgen05(ctypes.byref(d["desc"]), ctypes.byref(d["kv"]), 0x5000, None, 0x8000, None, 4, 0,
                                          0x10000, 1 << 30, None, None) == UNSUPPORTED


def test_binding_checks_shapes_before_it_calls():
    import paper_2602_11937_b200 as P
    d = P.layer_desc(kv_dtype=P.KV_FP4_E2M1)
    x = torch.zeros(2, 3, 8, 64, dtype=torch.bfloat16)
    q = torch.zeros(2, 3, 64, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="go together"):
        P.puzzle_kv_append_rope(d, P.KVView(), P.Rope(), q, x, x, None)
    with pytest.raises(ValueError, match="v_new must be"):
        P.puzzle_kv_append_rope(d, P.KVView(), P.Rope(), None, x, x[:, :2], None)
    with pytest.raises(ValueError, match="CUDA tensor"):
        P.puzzle_kv_append_rope(d, P.KVView(), P.Rope(), None, x, x, None)
    with pytest.raises(ValueError, match="v_out must be"):
        P.puzzle_kv_read_tokens(d, P.KVView(), x, x[:1])
    with pytest.raises(ValueError, match="CUDA tensor"):
        P.rope_view(torch.zeros(4, 64))


@pytest.mark.parametrize("n_new", [1, 2])
def test_more_heads_than_a_grid_dimension_holds_are_refused(n_new):
    heads = dict(num_q_heads=8 * 4097, desc__num_kv_heads=4097)
    wide = dict(heads, qkv__q_seq_stride=1 << 30, qkv__q_token_stride=1 << 24)
    assert _append(**wide, n_new=n_new) == UNSUPPORTED
    lib, d = _args(**heads, n_new=n_new)
    desc, kv = ctypes.byref(d["desc"]), ctypes.byref(d["kv"])
    assert lib.puzzle_kv_append(desc, kv, 0x6000, 0x7000, 4, None, None) == UNSUPPORTED
    assert lib.puzzle_kv_append_tokens(desc, kv, 0x6000, 0x7000, None, 4, n_new, None, None) == UNSUPPORTED
    assert lib.puzzle_kv_read_tokens(desc, kv, 0x9000, 0xA000, None, 4, n_new, None, None) == UNSUPPORTED


def test_binding_refuses_tensors_of_another_device(monkeypatch):
    """A kernel is launched on the current device; the memory of another one is not its to read."""
    from paper_2602_11937_b200 import binding as B

    class Elsewhere:
        def get_device(self):
            return 1
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    with pytest.raises(ValueError, match="the tensors are on cuda:1, the current device is cuda:0"):
        B._stream(None, Elsewhere())
