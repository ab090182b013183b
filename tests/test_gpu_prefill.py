"""The operators as they are used together: packed prompts through a stack of full and window layers (append with rotation,
attention, the window layers on rings of blocks), pieces behind them, then decode steps, for every cache type."""
import pytest
import torch

import paper_2602_11937_b200 as P
from prompt_helpers import BLOCK, D, FLOOR, KINDS, WEIGHT, attention64, cached, check, gen, make_cache, make_starts

pytestmark = pytest.mark.gpu
WINDOWS, HQ, HKV, BLOCKS = [0, 40, 17], 64, 8, 24
ALL = ("fp8", "bf16", "fp4")


class Model:
    def __init__(self, kv, lens, rings, rotate=True, seed=2):
        g = gen(seed)
        self.kv, self.batch = kv, len(lens)
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.scales = [[(0.01 + 0.01 * torch.rand(HKV, generator=g, device="cuda")) for _ in "kv"] for _ in WINDOWS]
        self.sinks = [torch.randn(HQ, generator=g, device="cuda") for _ in WINDOWS]
        self.caches, self.tables = [], []
        for w in WINDOWS:
            ring = rings and w
            nb = self.batch * (P.window_ring_blocks(w) if ring else BLOCKS)
            self.caches.append(make_cache(kv, nb, HKV, g))
            self.tables.append((P.ring_block_table(self.batch, w, BLOCKS) if ring else P.linear_block_table(self.batch, BLOCKS)).cuda())
        self.cos_sin = P.rope_table(BLOCKS * BLOCK).cuda()
        self.rope = P.rope_view(self.cos_sin) if rotate else None
        self.stack = P.DecodeStack(WINDOWS, [c[0] for c in self.caches], [c[1] for c in self.caches], self.lens, self.tables, BLOCKS,
                                   [s[0] for s in self.scales], [s[1] for s in self.scales], self.sinks, kv_dtype=KINDS[kv],
                                   rope=self.rope)

    def turned(self, rows, first):
        if self.rope is None:
            return rows
        pos = torch.arange(first, first + rows.shape[0], device="cuda")
        c, s = self.cos_sin[pos][:, None, :32], self.cos_sin[pos][:, None, 32:]
        x = rows.float()
        return torch.cat([x[..., :32] * c - x[..., 32:] * s, x[..., 32:] * c + x[..., :32] * s], -1).bfloat16()

    def keys(self, i, b, n):
        return [cached(self.kv, self.caches[i][j], self.scales[i][j], self.tables[i][b], 0, n, j == 1) for j in (0, 1)]


def parts(x):
    return [t[:, :HQ] for t in x], [t[:, HQ:HQ + HKV] for t in x], [t[:, HQ + HKV:] for t in x]


@pytest.mark.parametrize("kv", ALL)
@pytest.mark.parametrize("rotate", [True, False])
def test_prompts_then_steps(kv, rotate):
    g = gen(7)
    prompt = [33, 0, 150, 1]
    at, starts = make_starts(prompt)
    qkv = [torch.randn(at[-1], HQ + 2 * HKV, D, generator=g, device="cuda").bfloat16() for _ in WINDOWS]
    models = [Model(kv, prompt, rings, rotate) for rings in (False, True)]
    outs = []
    for m in models:
        out = [torch.empty(at[-1], HQ, D, dtype=torch.bfloat16, device="cuda") for _ in WINDOWS]
        m.stack.prefill(*parts(qkv), starts, out)
        torch.cuda.synchronize()
        assert m.stack.status.item() == 0
        outs.append(out)
    for i, w in enumerate(WINDOWS):
        assert torch.equal(outs[0][i], outs[1][i])
        for b, n in enumerate(prompt):
            if n:
                x = qkv[i][at[b]:at[b + 1]]
                q, k = models[0].turned(x[:, :HQ], 0), models[0].turned(x[:, HQ:HQ + HKV], 0)
                want, lse, size = attention64(q, k.double(), x[:, HQ + HKV:].double(), 0, w, models[0].sinks[i], 0.125)
                check("layer %d" % i, outs[0][i][at[b]:at[b + 1]], lse, want, lse, size, WEIGHT["packed"])
    # decode steps: the rings hold what the full caches hold of the windows
    for step in range(20):
        new = [torch.randn(4, HQ + 2 * HKV, D, generator=g, device="cuda").bfloat16() for _ in WINDOWS]
        got = []
        for m in models:
            m.lens += 1
            out = [torch.empty(4, HQ, D, dtype=torch.bfloat16, device="cuda") for _ in WINDOWS]
            q, k, v = parts(new)
            m.stack.step([x.contiguous() for x in q], [x.contiguous() for x in k], [x.contiguous() for x in v], out)
            got.append(out)
        torch.cuda.synchronize()
        for i, w in enumerate(WINDOWS):
            assert (got[0][i].double() - got[1][i].double()).abs().max() <= 2.0 ** -7
            if step in (0, 19):
                for b in range(4):
                    n = prompt[b] + step + 1
                    k, v = models[0].keys(i, b, n)
                    want, _, _ = attention64(models[0].turned(new[i][b:b + 1, :HQ], n - 1), k, v, n - 1, w, models[0].sinks[i], 0.125)
                    # bf16 rounding of outputs below 4, and the decode kernels' own bound
                    assert (got[0][i][b].double() - want[0]).abs().max() <= 2.0 ** -7 + 4e-3


@pytest.mark.parametrize("kv", ALL)
def test_pieces_behind_the_prompts(kv):
    """A prompt in three pieces: the first over its own keys, the others over the cache."""
    g = gen(9)
    m = Model(kv, [0, 0], False)
    sizes = [[40, 17], [100, 1], [33, 60]]
    done = [0, 0]
    for piece, new in enumerate(sizes):
        at, starts = make_starts(new)
        qkv = [torch.randn(at[-1], HQ + 2 * HKV, D, generator=g, device="cuda").bfloat16() for _ in WINDOWS]
        m.lens += torch.tensor(new, dtype=torch.int32, device="cuda")
        out = [torch.empty(at[-1], HQ, D, dtype=torch.bfloat16, device="cuda") for _ in WINDOWS]
        stream = torch.cuda.Stream() if piece == 1 else None
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        m.stack.prefill(*parts(qkv), starts, out, continued=piece > 0, stream=stream)
        torch.cuda.synchronize()
        assert m.stack.status.item() == 0
        for i, w in enumerate(WINDOWS):
            for b, n in enumerate(new):
                if piece == 0:
                    continue
                total = done[b] + n
                lo = max(0, done[b] + 1 - w) if w else 0
                k, v = m.keys(i, b, total)
                q = m.turned(qkv[i][at[b]:at[b + 1], :HQ], done[b])
                if lo:                       # of the first piece a window layer keeps what later tokens see
                    k[:lo], v[:lo] = 0, 0
                want, lse, size = attention64(q, k, v, done[b], w, m.sinks[i], 0.125, FLOOR[kv])
                check("layer %d" % i, out[i][at[b]:at[b + 1]], lse, want, lse, size, WEIGHT[kv])
        done = [a + b for a, b in zip(done, new)]


def test_prompt_attention_in_a_graph():
    """Append and both attentions captured, replayed with other tokens and other lengths."""
    g = gen(4)
    m = Model("fp8", [64, 96], False)
    desc, view = m.stack.descs[0], m.stack.views[0]
    qkv = torch.randn(160, HQ + 2 * HKV, D, generator=g, device="cuda").bfloat16()
    starts = make_starts([64, 96])[1]
    q, k = torch.empty(160, HQ, D, dtype=torch.bfloat16, device="cuda"), torch.empty(160, HKV, D, dtype=torch.bfloat16, device="cuda")
    out = [torch.empty_like(q) for _ in range(2)]
    ws = torch.empty(P.puzzle_chunk_attn_workspace_bytes(desc, 2, 160), dtype=torch.uint8, device="cuda")

    def run():
        P.puzzle_kv_append_packed(desc, view, m.rope, qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], starts, q, k)
        P.puzzle_prompt_attn(desc, q, k, qkv[:, HQ + HKV:], starts, m.sinks[0], out[0])
        P.puzzle_chunk_attn(desc, view, q, starts, m.sinks[0], out[1], workspace=ws)
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for new in ([64, 96], [1, 130], [100, 0]):
        qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda"))
        at, s = make_starts(new)
        starts.copy_(s)
        m.lens.copy_(torch.tensor(new, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for b, n in enumerate(new):
            if n:
                x = qkv[at[b]:at[b + 1]]
                qq, kk = m.turned(x[:, :HQ], 0), m.turned(x[:, HQ:HQ + HKV], 0)
                want, lse, size = attention64(qq, kk.double(), x[:, HQ + HKV:].double(), 0, 0, m.sinks[0], 0.125)
                check("prompt", out[0][at[b]:at[b + 1]], lse, want, lse, size, WEIGHT["packed"])
                kc, vc = m.keys(0, b, n)
                want, lse, size = attention64(qq, kc, vc, 0, 0, m.sinks[0], 0.125, FLOOR["fp8"])
                check("chunk", out[1][at[b]:at[b + 1]], lse, want, lse, size, WEIGHT["fp8"])
