"""The operators as they are used together: a prompt chunk appended with the rotation and read back, causal attention of
its last tokens, then decode steps of a stack of layers (full and window layers, the latter on rings of blocks) in a
captured graph, against the plain references and the float64 oracle, for every cache type."""
import numpy as np
import pytest
import torch

import oracle
from helpers import bf16_bits, bits_to_bf16
import kv_reference as R

pytestmark = pytest.mark.gpu

WINDOWS, BATCH, HQ, HKV, BLOCKS = [0, 40, 17], 2, 64, 8, 6


@pytest.mark.parametrize("kind", ["fp8", "bf16", "fp4"])
def test_prompt_then_steps(kind):
    import paper_2602_11937_b200 as P
    dtype = {"fp8": R.FP8, "bf16": R.BF16, "fp4": R.FP4}[kind]
    r = np.random.default_rng(3)
    g = torch.Generator().manual_seed(5)
    draw = lambda *shape: torch.randn(*shape, generator=g).clamp(-4, 4).to(torch.bfloat16)
    prompt = np.array([33, 20], np.int32)                     # tokens of each sequence's chunk
    n_chunk, steps = 33, 12
    cos_sin = P.rope_table(200, 64, theta=10000.0)
    table_dev = cos_sin.cuda()
    rope = P.rope_view(table_dev)
    lens = torch.from_numpy(prompt.copy()).cuda()
    scale = [tuple((0.01 + 0.01 * r.random(HKV)).astype(np.float32) for _ in "kv") for _ in WINDOWS]
    sinks = [r.standard_normal(HQ).astype(np.float32) for _ in WINDOWS]
    # the prompt goes through tables that keep every block; window layers then move to their rings by appending the
    # visible tail again (same bytes: appends are deterministic)
    ref, dev, linear = [], [], P.linear_block_table(BATCH, BLOCKS).numpy()
    for i, w in enumerate(WINDOWS):
        c = R.Cache(dtype, BATCH * BLOCKS, HKV, i)
        ref.append(c)
        up = (lambda a: bits_to_bf16(a).cuda()) if dtype == R.BF16 else (lambda a: torch.from_numpy(a.copy()).cuda())
        nb = BATCH * BLOCKS if w == 0 else BATCH * P.window_ring_blocks(w)
        table = P.linear_block_table(BATCH, BLOCKS) if w == 0 else P.ring_block_table(BATCH, w, BLOCKS)
        dev.append(dict(k=up(c.k[:nb]), v=up(c.v[:nb]), table=table.cuda(), ks=torch.from_numpy(scale[i][0]).cuda(),
                        vs=torch.from_numpy(scale[i][1]).cuda(), sinks=torch.from_numpy(sinks[i]).cuda()))
    lens_np = prompt.copy()
    qkv = [draw(BATCH, n_chunk, HQ + 2 * HKV, 64) for _ in WINDOWS]
    cut = lambda t: (t[..., :HQ, :], t[..., HQ:HQ + HKV, :], t[..., HQ + HKV:, :])
    new = torch.from_numpy(prompt).cuda()
    for i, w in enumerate(WINDOWS):
        d = dev[i]
        desc = P.layer_desc(window=w, kv_dtype=dtype)
        view = P.kv_view(d["k"], d["v"], lens, block_table=d["table"], k_scale=d["ks"], v_scale=d["vs"])
        q, k, v = cut(qkv[i].cuda())
        hq, hk, hv = (bf16_bits(x) for x in cut(qkv[i]))
        want_q = R.append(ref[i], linear, BLOCKS, lens_np, prompt, hq, hk, hv, *scale[i], cos_sin.numpy())
        if w:                                                 # a ring holds 16 (R - 1) tokens of a call at most
            keep = min(n_chunk, 16 * (P.window_ring_blocks(w) - 1))
            for b in range(BATCH):                            # each sequence's tail on its own
                t0 = max(0, int(prompt[b]) - keep)
                one = P.kv_view(d["k"], d["v"], lens[b:b + 1], block_table=d["table"][b:b + 1], k_scale=d["ks"],
                                v_scale=d["vs"])
                q_out = torch.empty(1, int(prompt[b]) - t0, HQ, 64, dtype=torch.bfloat16, device="cuda")
                P.puzzle_kv_append_rope(desc, one, rope, q[b:b + 1, t0:prompt[b]], k[b:b + 1, t0:prompt[b]],
                                        v[b:b + 1, t0:prompt[b]], q_out)
                assert np.array_equal(bf16_bits(q_out)[0], want_q[b, t0:prompt[b]])
            continue
        q_out = torch.full((BATCH, n_chunk, HQ, 64), 3.0, dtype=torch.bfloat16, device="cuda")
        P.puzzle_kv_append_rope(desc, view, rope, q, k, v, q_out, new_lens=new)
        back = {x: torch.zeros(BATCH, n_chunk, HKV, 64, dtype=torch.bfloat16, device="cuda") for x in "kv"}
        P.puzzle_kv_read_tokens(desc, view, back["k"], back["v"], read_lens=new)
        torch.cuda.synchronize()
        for b in range(BATCH):
            assert np.array_equal(bf16_bits(q_out)[b, :prompt[b]], want_q[b, :prompt[b]])
            for t in range(prompt[b]):
                for x, s in zip("kv", scale[i]):
                    raw = np.stack([ref[i].get(linear[b, t // 16], t % 16, h, x == "v") for h in range(HKV)])
                    want = raw if dtype == R.BF16 else raw.astype(np.float32) * s[:, None]
                    assert np.array_equal(bf16_bits(back[x])[b, t], R.round_bf16(np.asarray(want, np.float32)))
        if dtype != R.BF16:                                   # the last three prompt tokens attend causally
            nq = 3
            ws = torch.empty(P.puzzle_decode_attn_tokens_workspace_bytes(desc, BATCH, nq), dtype=torch.uint8, device="cuda")
            P.puzzle_decode_attn_tokens_workspace_init(desc, BATCH, nq, ws)
            last = torch.stack([q_out[b, prompt[b] - nq:prompt[b]] for b in range(BATCH)])
            out = torch.empty_like(last)
            P.puzzle_decode_attn_tokens(desc, view, last, d["sinks"], out, workspace=ws)
            torch.cuda.synchronize()
            for j in range(nq):
                _check(ref[i], linear, lens_np - nq + 1 + j, scale[i], bf16_bits(last[:, j].contiguous()), sinks[i], w,
                       out[:, j])
    # ---- decode steps through the stack, one graph replayed
    stack = P.DecodeStack(WINDOWS, [d["k"] for d in dev], [d["v"] for d in dev], lens, [d["table"] for d in dev], BLOCKS,
                          [d["ks"] for d in dev], [d["vs"] for d in dev], [d["sinks"] for d in dev], kv_dtype=dtype, rope=rope)
    buf = [torch.zeros(BATCH, HQ + 2 * HKV, 64, dtype=torch.bfloat16, device="cuda") for _ in WINDOWS]
    q, k, v = ([cut(b)[j] for b in buf] for j in range(3))
    out = [torch.empty(BATCH, HQ, 64, dtype=torch.bfloat16, device="cuda") for _ in WINDOWS]
    lens.add_(1)                                              # capture() runs the step once: on the first step's data
    first = [draw(BATCH, HQ + 2 * HKV, 64) for _ in WINDOWS]
    for b, x in zip(buf, first):
        b.copy_(x)
    graph = stack.capture(q, k, v, out)
    for step in range(steps):
        if step:
            lens.add_(1)
            first = [draw(BATCH, HQ + 2 * HKV, 64) for _ in WINDOWS]
            for b, x in zip(buf, first):
                b.copy_(x)
        for o in out:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        lens_np = lens_np + 1
        for i, w in enumerate(WINDOWS):
            hq, hk, hv = (bf16_bits(x)[:, None] for x in cut(first[i]))
            rotated = R.append(ref[i], linear, BLOCKS, lens_np, None, hq, hk, hv, *scale[i], cos_sin.numpy())
            _check(ref[i], linear, lens_np, scale[i], rotated[:, 0], sinks[i], w, out[i])
    assert int(stack.status.item()) == 0


def _check(cache, table, lens, scale, q_bits, sinks, window, out):
    """The framework's bound for decode attention (2e-3, and half a bf16 step from magnitude 1 on); the 4-bit kernels'
    P is rounded to f16, 2^-11 of an output below 2 in magnitude: 1e-3 more."""
    ref, _ = oracle.decode_attn(cache.k, cache.v, cache.kind, table, BLOCKS, np.asarray(lens, np.int32), scale[0], scale[1],
                                q_bits, sinks, window, 0.125)
    got = out.double().cpu().numpy().reshape(ref.shape)
    bound = 2e-3 + 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 * 2.0 if cache.kind == R.FP4 else 0.0)
    assert (np.abs(got - ref) <= bound).all(), float((np.abs(got - ref) - bound).max())
