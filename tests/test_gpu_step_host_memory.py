"""The step from host memory, over every way q, k_new and v_new can lie there: in one pinned buffer one behind the other (one copy),
in pinned buffers of their own that happen to follow each other (a copy may not cross from one into the next), and apart."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BATCH, CONTEXT = 16, 300                # q 128 KiB, k and v 16 KiB: whole pages, so that buffers of their own can touch


def _one_buffer():
    x = torch.empty(BATCH * 80 * 64, dtype=torch.bfloat16).pin_memory()
    cut = [BATCH * 64 * 64, BATCH * 8 * 64, BATCH * 8 * 64]
    return list(x.split(cut)), lambda: None


def _neighbours():
    """One allocation, its three parts page-locked each on its own."""
    page, sizes = 4096, [BATCH * 64 * 64 * 2, BATCH * 8 * 64 * 2, BATCH * 8 * 64 * 2]
    raw = torch.empty(sum(sizes) + page, dtype=torch.uint8)
    at = -raw.data_ptr() % page
    rt, parts = torch.cuda.cudart(), []
    for n in sizes:
        part = raw[at:at + n]
        assert int(rt.cudaHostRegister(part.data_ptr(), n, 0)) == 0
        parts.append(part)
        at += n

    def release():
        torch.cuda.synchronize()
        for part in parts:
            assert int(rt.cudaHostUnregister(part.data_ptr())) == 0
    return [part.view(torch.bfloat16) for part in parts], release


def _own_buffers():
    return [torch.empty(BATCH * h * 64, dtype=torch.bfloat16).pin_memory() for h in (64, 8, 8)], lambda: None


def _pageable():
    return list(torch.empty(BATCH * 80 * 64, dtype=torch.bfloat16).split([BATCH * 64 * 64, BATCH * 8 * 64, BATCH * 8 * 64])), \
        lambda: None


@pytest.mark.parametrize("kv_dtype", [0, 1, 2])
@pytest.mark.parametrize("place", [_one_buffer, _neighbours, _own_buffers, _pageable])
def test_inputs_wherever_they_lie(place, kv_dtype):
    import paper_2602_11937_b200 as P
    shape = {0: (16, 64), 1: (16, 64), 2: (576,)}[kv_dtype]
    blocks = -(-CONTEXT // 16)
    new = lambda: [torch.zeros(BATCH * blocks, 8, *shape, dtype=torch.bfloat16 if kv_dtype == 1 else torch.uint8, device="cuda")
                   for _ in range(2)]
    lens = torch.full((BATCH,), CONTEXT, dtype=torch.int32, device="cuda")
    scale = torch.full((8,), 0.01, device="cuda")
    d = P.layer_desc(kv_dtype=kv_dtype)
    g = torch.Generator().manual_seed(kv_dtype)
    values = [torch.randn(BATCH, h, 64, generator=g).to(torch.bfloat16) for h in (64, 8, 8)]
    ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(d, BATCH), dtype=torch.uint8, device="cuda")
    P.puzzle_decode_attn_workspace_init(d, BATCH, ws)
    here, there = new(), new()
    view = P.kv_view(*here, lens, max_blocks_per_seq=blocks, k_scale=scale, v_scale=scale)
    want = torch.empty(BATCH, 64, 64, dtype=torch.bfloat16, device="cuda")
    P.puzzle_kv_append(d, view, values[1].cuda(), values[2].cuda())
    P.puzzle_decode_attn(d, view, values[0].cuda(), None, want, workspace=ws)
    view = P.kv_view(*there, lens, max_blocks_per_seq=blocks, k_scale=scale, v_scale=scale)
    host, release = place()
    host = [t.view(v.shape).copy_(v) for t, v in zip(host, values)]
    out = torch.zeros(BATCH, 64, 64, dtype=torch.bfloat16).pin_memory()
    staging = torch.empty(P.puzzle_decode_step_host_staging_bytes(d, BATCH), dtype=torch.uint8, device="cuda")
    P.puzzle_decode_step_host(d, view, *host, None, out, staging, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(here, there))
    # the same kernel on the same bytes: the order of float32 sums, one bf16 step
    assert torch.allclose(out.float(), want.cpu().float(), rtol=2.0 ** -7, atol=2.0 ** -20)
    release()
