"""Argument errors of the entry points for packed tokens: found on the host before anything is launched, so they are tested
without a GPU (the pointers are never followed)."""
import ctypes

import pytest
import torch

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4
ref = lambda x: ctypes.byref(x) if x is not None else None


def _args(over):
    from paper_2602_11937_b200 import binding as B
    desc = B.layer_desc(kv_dtype=over.pop("kv_dtype", 0),
                        **{k: over.pop(k) for k in ("window", "head_dim", "num_q_heads", "num_kv_heads", "block_size") if k in over})
    kv = B.KVView()
    kv.k_cache, kv.v_cache, kv.seq_lens = 0x1000, 0x2000, 0x3000
    kv.num_blocks, kv.max_blocks_per_seq = 64, 16
    rope = B.Rope(0x4000, 1024, 64, 0, None)
    qkv = B.QKV(0x5000, 0x6000, 0x7000, 0, 4096, 0, 512, 0, 512)
    d = dict(desc=desc, kv=kv, rope=rope, qkv=qkv, q_out=0x8000, k_out=0x9000, starts=0xA000, batch=4, total=9, keep=0, out=0x8000,
             workspace=0x10000, workspace_bytes=1 << 30, stride=4096)
    for k, v in over.items():
        where, _, field = k.partition("__")
        if field:
            setattr(d[where], field, v)
        else:
            d[k] = v
    return B._load(), d


COMMON = [
    (dict(desc=None), NULL), (dict(starts=None), NULL), (dict(head_dim=128), UNSUPPORTED), (dict(num_q_heads=32), UNSUPPORTED),
    (dict(block_size=32), UNSUPPORTED), (dict(window=-1), SHAPE), (dict(kv_dtype=3), SHAPE), (dict(batch=0), SHAPE),
    (dict(batch=5000), UNSUPPORTED), (dict(total=-1), SHAPE), (dict(total=(1 << 30) + 1), SHAPE),
]


@pytest.mark.parametrize("over, want", COMMON + [
    (dict(kv=None), NULL), (dict(qkv=None), NULL), (dict(rope__cos_sin=None), NULL), (dict(qkv__k=None), NULL),
    (dict(qkv__v=None), NULL), (dict(q_out=None), NULL), (dict(rope=None), SHAPE), (dict(kv__num_blocks=63), SHAPE),
    (dict(rope=None, qkv__q=None, q_out=None), SHAPE), (dict(rope__rotary_dim=24), UNSUPPORTED),
    (dict(rope__rotary_dim=80), SHAPE), (dict(rope__num_positions=0), SHAPE), (dict(rope__cos_sin=0x4008), SHAPE),
    (dict(qkv__q=0x5008), SHAPE), (dict(qkv__k=0x6008), SHAPE), (dict(qkv__v=0x7002), SHAPE), (dict(q_out=0x8008), SHAPE),
    (dict(k_out=0x9004), SHAPE), (dict(qkv__k_token_stride=508), SHAPE), (dict(qkv__v_token_stride=0), SHAPE),
    (dict(qkv__q_token_stride=4100), SHAPE), (dict(qkv__q_token_stride=-4096), SHAPE),
    (dict(q_out=0x5000, qkv__q_token_stride=5120), SHAPE), (dict(k_out=0x6000, qkv__k_token_stride=5120), SHAPE),
    (dict(num_q_heads=8 * 4097, num_kv_heads=4097), UNSUPPORTED), (dict(total=0, qkv__k=None), OK), (dict(keep=-1), SHAPE),
])
def test_append_packed(over, want):
    lib, d = _args(dict(over))
    assert lib.puzzle_kv_append_packed(ref(d["desc"]), ref(d["kv"]), ref(d["rope"]), ref(d["qkv"]), d["q_out"], d["k_out"],
                                       d["starts"], d["batch"], d["total"], d["keep"], None, None) == want


@pytest.mark.parametrize("over, want", COMMON + [
    (dict(qkv=None), NULL), (dict(qkv__q=None), NULL), (dict(qkv__k=None), NULL), (dict(qkv__v=None), NULL),
    (dict(out=None), NULL), (dict(qkv__q=0x5008), SHAPE), (dict(qkv__k=0x6008), SHAPE), (dict(qkv__v=0x7002), SHAPE),
    (dict(out=0x8004), SHAPE), (dict(qkv__k_token_stride=508), SHAPE), (dict(qkv__v_token_stride=504), SHAPE),
    (dict(qkv__q_token_stride=4100), SHAPE), (dict(qkv__q_token_stride=1 << 39), SHAPE), (dict(total=0, out=None), OK),
])
def test_prompt_attn(over, want):
    lib, d = _args(dict(over))
    assert lib.puzzle_prompt_attn(ref(d["desc"]), ref(d["qkv"]), d["starts"], None, d["out"], None, d["batch"], d["total"],
                                  None, None) == want


@pytest.mark.parametrize("over, want", COMMON + [
    (dict(kv=None), NULL), (dict(kv__seq_lens=None), NULL), (dict(q=None), NULL), (dict(out=None), NULL), (dict(q=0x5008), SHAPE),
    (dict(out=0x8008), SHAPE), (dict(stride=4100), SHAPE), (dict(stride=4088), SHAPE), (dict(workspace=None), WORKSPACE),
    (dict(workspace=0x10008), WORKSPACE), (dict(workspace_bytes=15), WORKSPACE), (dict(kv__k_cache=0x1008), SHAPE),
    (dict(kv__max_blocks_per_seq=(1 << 26) + 1), UNSUPPORTED), (dict(total=0, q=None), OK),
])
def test_chunk_attn(over, want):
    over = dict(over)
    q = over.pop("q", 0x5000)
    lib, d = _args(over)
    assert lib.puzzle_chunk_attn(ref(d["desc"]), ref(d["kv"]), q, d["stride"], d["starts"], None, d["out"], None, d["batch"],
                                 d["total"], d["workspace"], d["workspace_bytes"], None, None) == want


def test_workspace_size():
    import paper_2602_11937_b200 as P
    d = P.layer_desc()
    size = lambda b, t: P.puzzle_chunk_attn_workspace_bytes(d, b, t)
    assert all(0 < size(b, t) < 90 << 20 for b in (1, 3, 64, 4096) for t in (0, 1, 5, 64, 600, 5000, 100000))
    assert size(1, 1 << 20) == 16               # many tokens: nothing is cut
    assert size(0, 1) == 0 and size(1, -1) == 0 and P.puzzle_chunk_attn_workspace_bytes(P.layer_desc(head_dim=128), 1, 1) == 0


def test_binding_checks_shapes_before_it_calls():
    import paper_2602_11937_b200 as P
    d = P.layer_desc()
    q, k = torch.zeros(5, 64, 64, dtype=torch.bfloat16), torch.zeros(5, 8, 64, dtype=torch.bfloat16)
    starts = torch.zeros(3, dtype=torch.int32)
    for bad, text in ((dict(q=q[:4], out=q[:4]), "k must be"), (dict(k=q), "k must be"), (dict(v=k[:, :, :32]), "v must be"),
                      (dict(starts=starts[:1]), "one element more"), (dict(q=q[0]), "q must be"), (dict(), "CUDA tensor")):
        a = dict(dict(q=q, k=k, v=k, starts=starts, sinks=None, out=q), **bad)
        with pytest.raises(ValueError, match=text):
            P.puzzle_prompt_attn(d, **a)
    with pytest.raises(ValueError, match="workspace tensor is required"):
        P.puzzle_chunk_attn(d, P.KVView(), q, starts, None, q)
    with pytest.raises(ValueError, match="go together"):
        P.puzzle_kv_append_packed(d, P.KVView(), P.Rope(), q, k, k, starts)
    with pytest.raises(ValueError, match="v_new must be"):
        P.puzzle_kv_append_packed(d, P.KVView(), None, None, k, k[:3], starts)
