"""The native module behind the hot entry points of the binding: what it refuses, without a GPU."""
import ctypes

import pytest
import torch


def _module():
    from paper_2602_11937_b200 import binding
    return binding._native(), binding


def test_descriptors_are_copied_byte_for_byte_or_refused():
    call, B = _module()
    x = torch.zeros(2, 8, 64, dtype=torch.bfloat16)
    desc, view = B.layer_desc(), B.KVView()
    assert (ctypes.sizeof(B.LayerDesc), ctypes.sizeof(B.KVView), ctypes.sizeof(B.Rope)) == (28, 64, 32)
    with pytest.raises(ValueError, match="descriptor has the wrong size"):
        call.kv_append(view, view, x, x, None, None)
    with pytest.raises(ValueError, match="descriptor has the wrong size"):
        call.kv_append(desc, desc, x, x, None, None)
    with pytest.raises(TypeError):
        call.kv_append(None, view, x, x, None, None)
    with pytest.raises(ValueError, match="k_new must be a CUDA tensor"):
        call.kv_append(desc, view, x, x, None, None)


@pytest.mark.parametrize("name, wanted", [("kv_append", 6), ("kv_append_tokens", 7), ("kv_append_rope", 10),
                                          ("kv_read_tokens", 7), ("decode_attn", 10), ("decode_attn_tcgen05", 10),
                                          ("decode_attn_tokens", 10), ("bind", 7)])
def test_argument_counts(name, wanted):
    call, _ = _module()
    for n in (0, wanted - 1, wanted + 1):
        with pytest.raises(TypeError):
            getattr(call, name)(*[None] * n)


def test_what_is_not_a_tensor():
    call, B = _module()
    d, v = B.layer_desc(), B.KVView()
    with pytest.raises(TypeError, match="q must be a tensor, got list"):
        call.decode_attn(d, v, [1.0], None, None, None, 0, torch.zeros(4), None, None)
    with pytest.raises(TypeError, match="workspace must be a tensor, got NoneType"):
        call.decode_attn(d, v, torch.zeros(4), None, None, None, 0, None, None, None)
    import paper_2602_11937_b200 as P
    with pytest.raises(ValueError, match="workspace is required"):
        P.puzzle_decode_attn(d, v, torch.zeros(4), None, torch.zeros(4))
    with pytest.raises(ValueError, match="workspace tensor is required"):
        P.puzzle_decode_attn_tokens(d, v, torch.zeros(4), None, torch.zeros(4))


def test_a_missing_module_fails_loudly(monkeypatch):
    _, B = _module()
    monkeypatch.setattr(B, "_lib", None)
    monkeypatch.setattr(B, "_call", None)
    monkeypatch.setattr(B, "_CALL_PATH", "/nonexistent/_puzzle_call.so")
    for _ in range(2):
        with pytest.raises(RuntimeError, match="is missing: build it"):
            B._native()


@pytest.mark.gpu
def test_tensors_that_the_calls_refuse():
    import paper_2602_11937_b200 as P
    d = P.layer_desc(kv_dtype=P.KV_FP4_E2M1)
    cache = torch.zeros(4, 8, 576, dtype=torch.uint8, device="cuda")
    lens = torch.ones(2, dtype=torch.int32, device="cuda")
    view = P.kv_view(cache, cache.clone(), lens, max_blocks_per_seq=2)
    q = torch.zeros(2, 64, 64, dtype=torch.bfloat16, device="cuda")
    out, k = torch.empty_like(q), torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(P.puzzle_decode_attn_workspace_bytes(d, 2), dtype=torch.uint8, device="cuda")
    bad = {"q": q.float(), "sinks": torch.zeros(64, device="cuda", dtype=torch.float64), "out": q.float(),
           "lse_out": torch.zeros(2, 64, dtype=torch.int32, device="cuda"), "dev_status": torch.zeros(1, device="cuda")}
    for name, t in bad.items():
        args = dict(q=q, sinks=None, out=out, lse_out=None, workspace=ws, dev_status=None)
        args[name] = t
        with pytest.raises(ValueError, match="%s must be torch" % name):
            P.puzzle_decode_attn(d, view, **args)
    with pytest.raises(ValueError, match="q must be contiguous"):
        P.puzzle_decode_attn(d, view, q.transpose(0, 1), None, out, workspace=ws)
    with pytest.raises(ValueError, match="out must be a CUDA tensor"):
        P.puzzle_decode_attn(d, view, q, None, out.cpu(), workspace=ws)
    with pytest.raises(P.PuzzleError, match="workspace missing"):
        P.puzzle_decode_attn(d, view, q, None, out, workspace=ws[:64])
    with pytest.raises(P.PuzzleError, match="out-of-range"):
        P.puzzle_decode_attn(d, view, q, None, out, num_splits=-7, workspace=ws)
    rope = P.rope_view(P.rope_table(8, 64).cuda())
    with pytest.raises(ValueError, match=r"q must be \(2, 64, 64\), got \(2, 32, 64\)"):
        P.puzzle_kv_append_rope(d, view, rope, q[:, :32], k, k, out)
    with pytest.raises(ValueError, match="heads of a token of k_new must be contiguous"):
        P.puzzle_kv_append_rope(d, view, rope, None, k.transpose(1, 2).contiguous().transpose(1, 2), k)
    with pytest.raises(ValueError, match="v_new must be a bf16 CUDA tensor"):
        P.puzzle_kv_append_rope(d, view, rope, None, k, k.float())
    with pytest.raises(ValueError, match="new_lens must be torch.int32, got"):
        P.puzzle_kv_append_rope(d, view, rope, None, k, k, new_lens=lens.long())
    with pytest.raises(AttributeError):
        P.puzzle_kv_append(d, view, k, k, stream=object())
    torch.cuda.synchronize()
    assert int(cache.sum()) == 0


@pytest.mark.gpu
def test_tensors_too_small_for_the_call_are_refused():
    """Nothing is launched: the kernels would read or write past their ends."""
    import paper_2602_11937_b200 as P
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype, device="cuda")
    d = P.layer_desc(kv_dtype=P.KV_FP4_E2M1)
    cache, lens = z(4, 8, 576, dtype=torch.uint8), torch.ones(2, dtype=torch.int32, device="cuda")
    view = P.kv_view(cache, cache.clone(), lens, max_blocks_per_seq=2)
    q, k, f32, i32 = z(2, 64, 64), z(2, 8, 64), torch.float32, torch.int32
    before = P.puzzle_launch_count()
    ws = z(P.puzzle_decode_attn_workspace_bytes(d, 2), dtype=torch.uint8)
    good = dict(q=q, sinks=z(64, dtype=f32), out=z(2, 64, 64), lse_out=z(2, 64, dtype=f32), workspace=ws,
                dev_status=z(1, dtype=i32))
    for name, t in dict(q=z(2, 63, 64), sinks=z(63, dtype=f32), out=z(1, 64, 64), lse_out=z(2, 63, dtype=f32),
                        dev_status=z(0, dtype=i32)).items():
        with pytest.raises(ValueError, match="%s has [0-9]+ elements, the call needs [0-9]+" % name):
            P.puzzle_decode_attn(d, view, **{**good, name: t})
    q3, ws3 = z(2, 3, 64, 64), z(P.puzzle_decode_attn_tokens_workspace_bytes(d, 2, 3), dtype=torch.uint8)
    good = dict(q=q3, sinks=None, out=z(2, 3, 64, 64), lse_out=None, q_lens=lens, workspace=ws3)
    for name, t in dict(out=z(2, 2, 64, 64), lse_out=z(2, 2, 64, dtype=f32), q_lens=z(1, dtype=i32)).items():
        with pytest.raises(ValueError, match="%s has" % name):
            P.puzzle_decode_attn_tokens(d, view, **{**good, name: t})
    with pytest.raises(ValueError, match="v_new has 512 elements, the call needs 1024"):
        P.puzzle_kv_append(d, view, k, k[:1])
    with pytest.raises(ValueError, match="k_new has 1024 elements, the call needs 2048"):
        P.puzzle_kv_append_tokens(d, view, k.view(2, 2, 4, 64), z(2, 2, 8, 64))
    with pytest.raises(ValueError, match="new_lens has 1 elements"):
        P.puzzle_kv_append_rope(d, view, P.rope_view(P.rope_table(8).cuda()), None, k, k, new_lens=lens[:1])
    with pytest.raises(ValueError, match="read_lens has 1 elements"):
        P.puzzle_kv_read_tokens(d, view, z(2, 1, 8, 64), z(2, 1, 8, 64), read_lens=lens[:1])
    assert P.puzzle_launch_count() == before
