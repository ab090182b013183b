"""Every tensor of a call has to lie on the current device: the check itself (no GPU needed), and that each argument of each
call goes through it, with tensors that pretend to lie on a second GPU (they have no memory; nothing is launched)."""
import pytest
import torch


def test_the_comparison():
    from paper_2602_11937_b200 import binding as B
    call = B._native()
    assert call.check_device("q", 0, 0) == 0 and call.check_device("q", 3, 3) == 0
    with pytest.raises(ValueError, match="v_new is on cuda:1, the current device is cuda:0"):
        call.check_device("v_new", 1, 0)
    with pytest.raises(ValueError, match="sinks is on cuda:0, the current device is cuda:2"):
        call.check_device("sinks", 0, 2)


def _elsewhere(t):
    from torch._subclasses import fake_tensor
    with fake_tensor.FakeTensorMode():
        return torch.empty(t.shape, dtype=t.dtype, device="cuda:1")


@pytest.mark.gpu
def test_each_argument_of_each_call(monkeypatch):
    import paper_2602_11937_b200 as P
    from torch._subclasses import fake_tensor
    monkeypatch.setattr(fake_tensor, "init_gpu_context", lambda device: None)      # there is no second GPU to wake
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype, device="cuda")
    i32, f32, u8 = torch.int32, torch.float32, torch.uint8
    lens = torch.ones(2, dtype=i32, device="cuda")
    d4, d8 = P.layer_desc(kv_dtype=P.KV_FP4_E2M1), P.layer_desc()
    c4, c8 = z(4, 8, 576, dtype=u8), z(4, 8, 16, 64, dtype=u8)
    view, view8 = P.kv_view(c4, c4.clone(), lens, max_blocks_per_seq=2), P.kv_view(c8, c8.clone(), lens, max_blocks_per_seq=2)
    table = P.rope_table(64).cuda()
    rope = P.rope_view(table)
    q, k, st = z(2, 64, 64), z(2, 8, 64), z(1, dtype=i32)
    ws = z(P.puzzle_decode_attn_workspace_bytes(d4, 2), dtype=u8)
    wt = z(P.puzzle_decode_attn_tokens_workspace_bytes(d4, 2, 3), dtype=u8)
    attn = dict(q=q, sinks=z(64, dtype=f32), out=z(2, 64, 64), lse_out=z(2, 64, dtype=f32), workspace=ws, dev_status=st)
    calls = [
        (P.puzzle_kv_append, view, dict(k_new=k, v_new=k.clone(), dev_status=st)),
        (P.puzzle_kv_append_tokens, view, dict(k_new=z(2, 3, 8, 64), v_new=z(2, 3, 8, 64), new_lens=lens, dev_status=st)),
        (P.puzzle_kv_append_rope, view, dict(rope=rope, q=q, k_new=k, v_new=k.clone(), q_out=z(2, 64, 64), new_lens=lens,
                                             dev_status=st)),
        (P.puzzle_kv_read_tokens, view, dict(k_out=z(2, 3, 8, 64), v_out=z(2, 3, 8, 64), read_lens=lens, dev_status=st)),
        (P.puzzle_decode_attn, view, attn),
        (P.puzzle_decode_attn_tcgen05, view8, attn),
        (P.puzzle_decode_attn_tokens, view, dict(q=z(2, 3, 64, 64), sinks=attn["sinks"], out=z(2, 3, 64, 64),
                                                 lse_out=z(2, 3, 64, dtype=f32), q_lens=lens, workspace=wt, dev_status=st)),
    ]
    for f, v, good in calls:
        d = d8 if v is view8 else d4
        f(d, v, **good)
        torch.cuda.synchronize()
        before = P.puzzle_launch_count()
        for name, t in good.items():
            if name != "rope":
                with pytest.raises(ValueError, match="%s is on cuda:1, the current device is cuda:0" % name):
                    f(d, v, **{**good, name: _elsewhere(t)})
        assert P.puzzle_launch_count() == before
