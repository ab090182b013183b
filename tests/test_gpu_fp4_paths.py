"""The 4-bit cache on paths that its other tests do not take: the step from host memory, blocks beyond 4 GiB, calls on two
streams at once, and a decode step in a graph whose sequences grow between replays."""
import numpy as np
import pytest
import torch

from helpers import bf16_bits
import kv_reference as R
from test_gpu_fp4_attention import Case

pytestmark = pytest.mark.gpu


def _workspace(c, splits=0):
    ws = torch.empty(c.P.puzzle_decode_attn_workspace_bytes(c.desc, c.batch, splits), dtype=torch.uint8, device="cuda").fill_(0xFF)
    c.P.puzzle_decode_attn_workspace_init(c.desc, c.batch, ws)
    return ws


@pytest.mark.parametrize("splits", [0, -2, 3])
def test_step_from_host_memory(splits):
    lens = [700, 1, 17, 64]
    c = Case(lens, hkv=2, seed=31, poison=False).upload()
    g = torch.Generator().manual_seed(32)
    k, v = (torch.randn(len(lens), 2, 64, generator=g).to(torch.bfloat16).pin_memory() for _ in "kv")
    out = torch.zeros(len(lens), 16, 64, dtype=torch.bfloat16).pin_memory()
    staging = torch.empty(c.P.puzzle_decode_step_host_staging_bytes(c.desc, c.batch), dtype=torch.uint8, device="cuda")
    c.P.puzzle_decode_step_host(c.desc, c.view, c.q[:, 0].contiguous().pin_memory(), k, v, c.d["sinks"], out, staging,
                                _workspace(c, splits), num_splits=splits, dev_status=c.status)
    torch.cuda.synchronize()
    want = R.Cache(R.FP4, c.k.shape[0], 2, 0)
    want.k, want.v = c.k, c.v
    R.append(want, c.table, c.mb, c.lens, None, None, bf16_bits(k)[:, None], bf16_bits(v)[:, None], c.k_scale, c.v_scale)
    assert np.array_equal(c.d["k"].cpu().numpy(), c.k) and np.array_equal(c.d["v"].cpu().numpy(), c.v)
    c.check(out.double().numpy(), c.run(splits)[1])
    assert int(c.status.item()) == 0


@pytest.mark.parametrize("kind", ["fp8", "bf16", "fp4"])
def test_blocks_beyond_32_bit_offsets(kind):
    """The same chunk, read-back and decode step in a small cache and in blocks at the end of one of more than 4 GiB."""
    import paper_2602_11937_b200 as P
    dtype = {"fp8": P.KV_FP8_E4M3, "bf16": P.KV_BF16, "fp4": P.KV_FP4_E2M1}[kind]
    hkv, n, per_seq, batch = 8, 70, 6, 2
    shape = (hkv, 576) if kind == "fp4" else (hkv, 16, 64)
    cells = {"fp8": torch.uint8, "bf16": torch.bfloat16, "fp4": torch.uint8}[kind]
    per_block = int(np.prod(shape)) * (2 if kind == "bf16" else 1)
    many = (1 << 32) // per_block + 100                       # the last blocks lie past the first 4 GiB of each cache
    g = torch.Generator().manual_seed(7)
    q, k, v = (torch.randn(batch, n, h, 64, generator=g).to(torch.bfloat16).cuda() for h in (8 * hkv, hkv, hkv))
    lens = torch.tensor([n, n + 21], dtype=torch.int32, device="cuda")
    desc, table = P.layer_desc(kv_dtype=dtype), P.rope_table(200, 64).cuda()
    results = []
    for nb in (batch * per_seq, many):
        order = torch.arange(nb - 1, nb - 1 - batch * per_seq, -1, dtype=torch.int32).view(batch, per_seq).cuda()
        kc, vc = (torch.empty(nb, *shape, dtype=cells, device="cuda") for _ in "kv")
        for cache in (kc, vc):
            cache[-batch * per_seq:].zero_()
        view = P.kv_view(kc, vc, lens, block_table=order)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        q_rot, out = torch.empty_like(q), torch.empty(batch, 8 * hkv, 64, dtype=torch.bfloat16, device="cuda")
        back = [torch.empty_like(k), torch.empty_like(v)]
        P.puzzle_kv_append_rope(desc, view, P.rope_view(table), q, k, v, q_rot, dev_status=status)
        one = [x[:, -1] for x in (q, k, v)]                   # the last token once more, by the step kernel
        P.puzzle_kv_append_rope(desc, view, P.rope_view(table), *one, torch.empty_like(out), dev_status=status)
        P.puzzle_kv_read_tokens(desc, view, *back, dev_status=status)
        ws = torch.empty(P.puzzle_decode_attn_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
        P.puzzle_decode_attn_workspace_init(desc, batch, ws)
        P.puzzle_decode_attn(desc, view, q_rot[:, -1].contiguous(), None, out, workspace=ws, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        tail = [cache[-batch * per_seq:].cpu() for cache in (kc, vc)]
        results.append([x.cpu() for x in (q_rot, out, *back)] + [t.flip(0) for t in tail])
        del kc, vc, view
    for a, b in zip(*results):
        if a.dtype == torch.bfloat16:
            a, b = a.view(torch.int16), b.view(torch.int16)
        assert torch.equal(a, b)
    torch.cuda.empty_cache()


def test_calls_on_two_streams_at_once():
    cases = [Case([3000, 2000, 40], hkv=8, seed=50).upload(), Case([900, 1, 5000], hkv=8, seed=51, window=600).upload()]
    streams = [torch.cuda.Stream() for _ in cases]
    work = [(_workspace(c), torch.zeros(20, c.batch, c.hq, 64, dtype=torch.bfloat16, device="cuda"),
             c.d["q"][:, 0].contiguous()) for c in cases]
    want = [c.run() for c in cases]
    torch.cuda.synchronize()
    for i in range(20):
        for c, s, (ws, out, q) in zip(cases, streams, work):
            c.P.puzzle_decode_attn(c.desc, c.view, q, c.d["sinks"], out[i], None, workspace=ws, dev_status=c.status, stream=s)
    torch.cuda.synchronize()
    for c, (_, out, _), (ref, lse) in zip(cases, work, want):
        c.check(ref, lse)
        assert (out.double().cpu().numpy() == ref).all()      # whole pairs and even shares alike: the order of sums is fixed
        assert int(c.status.item()) == 0


def test_a_graph_whose_sequences_grow_between_replays():
    """What the host chooses from (the table's row length) holds for every replay; the lengths are read on the device."""
    c = Case([1, 500, 30], hkv=2, max_blocks=80, seed=60, poison=False).upload()
    ws, q = _workspace(c), c.d["q"][:, 0].contiguous()
    out = torch.zeros(c.batch, c.hq, 64, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(c.batch, c.hq, device="cuda")
    call = lambda: c.P.puzzle_decode_attn(c.desc, c.view, q, c.d["sinks"], out, lse, workspace=ws, dev_status=c.status)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lens in ([1, 500, 30], [0, 1280, 16], [1280, 0, 0], [640, 641, 639]):
        c.lens[:] = lens
        c.d["lens"].copy_(torch.from_numpy(c.lens))
        graph.replay()
        torch.cuda.synchronize()
        c.check(out.double().cpu().numpy(), lse.double().cpu().numpy())
