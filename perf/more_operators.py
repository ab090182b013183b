"""Operators of the prompt phase, as they are measured: attention over whole prompts, attention of chunks of new tokens over
the paged cache, and the append of packed tokens with their position rotation.

The tokens of several sequences lie packed, one row each: sequence b has rows starts[b] .. starts[b + 1] - 1 of every
array.  `run` with `own` false computes the plain forms in elementary torch operations; with `own` true it makes the calls a
user of the package makes.  64 query heads on 8 KV heads of 64 channels, caches paged in blocks of 16 tokens.

A query token at position p sees the keys [p + 1 - min(W, p + 1), p] (all of [0, p] without a window W); every query head
has a sink, one more column of its softmax that carries no value.
"""
import math
import random

import torch

own = False

HQ, HKV, D, BLOCK = 64, 8, 64, 16
GROUP = HQ // HKV
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------------------------------- cases ----

def listed():
    prompt = dict(op="prompt", window=0, ragged=True)
    chunk = dict(op="chunk", window=0, ragged=False)
    append = dict(op="append", interleaved=False, rotary=64, ragged=True, rotate=True)
    return [
        # one short question: nothing but latency
        dict(prompt, name="prompt_1x33", batch=1, tokens=33, ragged=False),
        # a serving batch of ragged prompts on a layer with a 128-token window
        dict(prompt, name="prompt_24x2000_w128", batch=24, tokens=2000, window=128),
        # the same on a full-context layer, fewer and longer
        dict(prompt, name="prompt_8x4001", batch=8, tokens=4001),
        # one long document
        dict(prompt, name="prompt_1x16384", batch=1, tokens=16384, ragged=False),
        # a few drafted tokens of one sequence at a short context: latency
        dict(chunk, name="chunk_fp8_1x5", kv="fp8", batch=1, tokens=5, context=777),
        # drafted tokens of a small batch at a long context: bound by the cache's bytes
        dict(chunk, name="chunk_fp8_8x12_32k", kv="fp8", batch=8, tokens=12, context=32768),
        # a piece of a long prompt behind what is cached already
        dict(chunk, name="chunk_fp8_1x512_64k", kv="fp8", batch=1, tokens=512, context=65536),
        # large ragged pieces over the 4-bit cache
        dict(chunk, name="chunk_fp4_3x2048_24k", kv="fp4", batch=3, tokens=2048, context=24001, ragged=True),
        # pieces and single tokens together over the bf16 cache, on a layer with a window
        dict(chunk, name="chunk_bf16_17x301_w500", kv="bf16", batch=17, tokens=301, context=9001, ragged=True, window=500),
        # a short prompt's tokens into the E4M3 cache: latency
        dict(append, name="append_fp8_1x20", kv="fp8", batch=1, tokens=20, ragged=False, context=20),
        # a serving batch of ragged prompts into the E4M3 cache
        dict(append, name="append_fp8_32x2048", kv="fp8", batch=32, tokens=2048, context=2048),
        # ragged pieces into the 4-bit cache, adjacent pairs rotated; the rounded tokens are read back
        dict(append, name="append_fp4_9x1500", kv="fp4", batch=9, tokens=1500, context=4100, interleaved=True, rotary=32),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("prompt", "prompt", "chunk", "chunk", "chunk", "append"))
    mix = rng.randrange(1 << 16)
    if op == "prompt":
        tokens = _log(rng, 1, 16384)
        batch = _log(rng, 1, max(1, min(64, 32768 // tokens, (1 << 28) // tokens ** 2)))
        return dict(op=op, batch=batch, tokens=tokens, window=rng.choice((0, 0, 128, _log(rng, 1, 8192))),
                    ragged=rng.random() < 0.6, mix=mix)
    kv = rng.choice(("fp8", "fp8", "fp4", "bf16"))
    if op == "chunk":
        tokens = _log(rng, 1, 4096)
        context = _log(rng, max(16, tokens), 65536)
        batch = _log(rng, 1, max(1, min(64, (1 << 26) // (tokens * context), (1 << 20) // context)))
        return dict(op=op, kv=kv, batch=batch, tokens=tokens, context=context,
                    window=rng.choice((0, 0, 0, 128, _log(rng, 1, 8192))), ragged=rng.random() < 0.6, mix=mix)
    tokens = _log(rng, 1, 4096)
    batch = _log(rng, 1, max(1, min(64, 32768 // tokens)))
    return dict(op=op, kv=kv, batch=batch, tokens=tokens, context=tokens + rng.randrange(0, 2048),
                interleaved=rng.random() < 0.3, rotary=rng.choice((64, 64, 32, 48)), ragged=rng.random() < 0.6,
                rotate=rng.random() < 0.85, mix=mix)


def _lens(case):
    """New tokens of every sequence and its length with them (which a server's program knows on its side)."""
    rng = random.Random(case.get("mix", 1) * 1009 + case["batch"] * 31 + case["tokens"])
    new, context = [], []
    for _ in range(case["batch"]):
        n, m = case["tokens"], case.get("context", case["tokens"])
        if case["ragged"]:
            # serving batches hold single tokens and nothing at all among their pieces
            n = rng.choice((0, 1, n)) if rng.random() < 0.15 else rng.randint(max(1, n // 4), n)
            if case["op"] != "prompt":
                m = rng.randint(max(1, n, m // 3), m)
        new.append(n)
        context.append(n if case["op"] == "prompt" else m)
    if sum(new) == 0:
        new[0], context[0] = 1, max(1, context[0])
    return new, context


# -------------------------------------------------------------------------------------------------- 4-bit format ----
# One (block, KV head) is 576 bytes: 512 of E2M1 codes, then 64 E4M3 scales, one per token and 16 channels.  K codes: token t
# at bytes 32 t .. 32 t + 31, channel d in byte d / 2 (even channel in the low nibble).  V codes: byte 256 (d / 32) +
# 32 (t / 2) + d % 32 (even token in the low nibble).  With b = d / 16 the scale of K is byte 16 b + 2 (t % 8) + t / 8 of
# the 64, that of V byte 16 b + 4 ((t % 8) / 2) + 2 (t / 8) + t % 2.

def _e4m3(x):
    """Float32 to the nearest E4M3 value, ties to even, saturating."""
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _quantise4(y):
    """y float32 [..., 64] (already divided by the head's scale) -> codes uint8 [..., 64], scales E4M3 [..., 4]."""
    g = y.unflatten(-1, (4, 16))
    t8 = _e4m3(g.abs().amax(-1) / 6.0)
    t = t8.float().unsqueeze(-1)
    a = (g / torch.where(t > 0, t, torch.ones_like(t))).abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = torch.where(t > 0, code + 8 * torch.signbit(g).to(torch.uint8), torch.zeros_like(code))
    return code.flatten(-2), t8


def _dequantise4(code, t8):
    """Codes uint8 [..., 64] and scales E4M3 [..., 4] -> float32 [..., 64], in units of the head's scale."""
    lut = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=code.device)
    return (lut[code.int()].unflatten(-1, (4, 16)) * t8.float().unsqueeze(-1)).flatten(-2)


def _pack4(code, t8, is_v):
    """Codes [nb][H][16][64], scales [nb][H][16][4] -> uint8 [nb][H][576]."""
    nb, h = code.shape[:2]
    s = t8.view(torch.uint8)
    if is_v:
        c = code.view(nb, h, 8, 2, 2, 32).permute(0, 1, 4, 2, 5, 3)             # half, token pair, channel, token
        s = s.view(nb, h, 2, 4, 2, 4).permute(0, 1, 5, 3, 2, 4)                 # 16 channels, pair, eighth, token
    else:
        c = code.view(nb, h, 16, 32, 2)
        s = s.view(nb, h, 2, 8, 4).permute(0, 1, 4, 3, 2)
    return torch.cat([(c[..., 0] | (c[..., 1] << 4)).reshape(nb, h, 512), s.reshape(nb, h, 64)], -1).contiguous()


def _unpack4(block, is_v):
    """uint8 [..., 576] -> codes [..., 16, 64], scales E4M3 [..., 16, 4]."""
    c, s = block[..., :512], block[..., 512:]
    lead = list(range(block.dim() - 1))
    n = len(lead)
    c = torch.stack([c & 15, c >> 4], -1)
    if is_v:
        c = c.unflatten(-2, (2, 8, 32)).permute(*lead, n + 1, n + 3, n, n + 2)  # token pair, token, half, channel
        s = s.unflatten(-1, (4, 4, 2, 2)).permute(*lead, n + 2, n + 1, n + 3, n)
    else:
        c = c.unflatten(-2, (16, 32))
        s = s.unflatten(-1, (4, 8, 2)).permute(*lead, n + 2, n + 1, n)
    return (c.reshape(*block.shape[:-1], 16, 64),
            s.reshape(*block.shape[:-1], 16, 4).contiguous().view(torch.float8_e4m3fn))


# ------------------------------------------------------------------------------------------------------- inputs ----

def _gen(seed, k):
    return torch.Generator(device="cuda").manual_seed((seed * 1000003 + k * 7919) & 0x7FFFFFFF)


def _fill(kv, nb, scale, seed, k, is_v):
    """A cache of nb blocks that holds N(0, 1) samples in the given type."""
    parts = []
    for lo in range(0, nb, 8192):
        x = torch.randn((min(8192, nb - lo), HKV, BLOCK, D), generator=_gen(seed, k + 100 + lo), device="cuda")
        y = x / scale[None, :, None, None]
        if kv == "fp4":
            parts.append(_pack4(*_quantise4(y), is_v))
        else:
            parts.append(x.bfloat16() if kv == "bf16" else _e4m3(y).view(torch.uint8))
    return torch.cat(parts)


def prepare(case, seed):
    op, batch = case["op"], case["batch"]
    g = _gen(seed, 1)
    new, context = _lens(case)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    total = starts[-1]
    s = {"case": case, "new": new, "context": context, "first": starts,
         "starts": torch.tensor(starts, dtype=torch.int32, device="cuda"),
         "lens": torch.tensor(context, dtype=torch.int32, device="cuda")}
    if op != "chunk":       # q, k and v are slices of one projection's output
        s["qkv"] = torch.randn(total, HQ + 2 * HKV, D, generator=g, device="cuda").bfloat16()
    if op != "append":
        s["q"] = s["qkv"][:, :HQ] if op == "prompt" else torch.randn(total, HQ, D, generator=g, device="cuda").bfloat16()
        s["sinks"] = torch.randn(HQ, generator=g, device="cuda")
        s["out"] = torch.zeros(total, HQ, D, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros(total, HQ, device="cuda")
    if op != "prompt":
        per_seq = -(-max(context) // BLOCK)
        nb = batch * per_seq
        s["per_seq"] = per_seq
        s["table"] = torch.randperm(nb, generator=g, device="cuda").to(torch.int32).view(batch, per_seq)
        # scales as a max calibration of N(0, 1) samples leaves them: about amax / 448, another for each head
        for k, name in enumerate(("k", "v")):
            s[name + "_scale"] = 0.008 + 0.004 * torch.rand(HKV, generator=g, device="cuda")
            s[name + "_cache"] = _fill(case["kv"], nb, s[name + "_scale"], seed, 10 + k, k == 1)
    if op == "append":
        if case["rotate"]:
            r, m = case["rotary"], max(context)
            angle = torch.arange(m, device="cuda", dtype=torch.float64)[:, None] * torch.pow(
                150000.0, -torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)
            s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], -1).float()
            s["q_out"] = torch.zeros(total, HQ, D, dtype=torch.bfloat16, device="cuda")
            s["k_out"] = torch.zeros(total, HKV, D, dtype=torch.bfloat16, device="cuda")
        if case["kv"] == "fp4":
            s["read_lens"] = torch.tensor(new, dtype=torch.int32, device="cuda")
            s["k_read"] = torch.zeros(batch, max(new), HKV, D, dtype=torch.bfloat16, device="cuda")
            s["v_read"] = torch.zeros_like(s["k_read"])
    if own:  # the descriptors and the workspace, which a program makes once per layer
        _plan(s)
    return s


def _plan(s):
    import paper_2602_11937_b200 as P
    case = s["case"]
    kinds = {"fp8": P.KV_FP8_E4M3, "bf16": P.KV_BF16, "fp4": P.KV_FP4_E2M1}
    s["desc"] = P.layer_desc(window=case.get("window", 0), kv_dtype=kinds[case.get("kv", "bf16")])
    if case["op"] == "prompt":
        return
    s["view"] = P.kv_view(s["k_cache"], s["v_cache"], s["lens"], block_table=s["table"], k_scale=s["k_scale"],
                          v_scale=s["v_scale"])
    if case["op"] == "chunk":
        size = P.puzzle_chunk_attn_workspace_bytes(s["desc"], case["batch"], s["first"][-1])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    else:
        s["rope"] = P.rope_view(s["cos_sin"], interleaved=case["interleaved"]) if case["rotate"] else None


# --------------------------------------------------------------------------------------------------------- run ----

def run(s):
    op = s["case"]["op"]
    if own:
        return {"prompt": _own_prompt, "chunk": _own_chunk, "append": _own_append}[op](s)
    return {"prompt": _plain_prompt, "chunk": _plain_chunk, "append": _plain_append}[op](s)


def _own_prompt(s):
    import paper_2602_11937_b200 as P
    qkv = s["qkv"]
    P.puzzle_prompt_attn(s["desc"], s["q"], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], s["starts"], s["sinks"], s["out"],
                         s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_chunk(s):
    import paper_2602_11937_b200 as P
    P.puzzle_chunk_attn(s["desc"], s["view"], s["q"], s["starts"], s["sinks"], s["out"], s["lse"],
                        workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_append(s):
    import paper_2602_11937_b200 as P
    qkv, rotate = s["qkv"], s["case"]["rotate"]
    k, v = qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]
    if rotate:
        P.puzzle_kv_append_packed(s["desc"], s["view"], s["rope"], qkv[:, :HQ], k, v, s["starts"], s["q_out"], s["k_out"])
    else:
        P.puzzle_kv_append_packed(s["desc"], s["view"], None, None, k, v, s["starts"])
    out = {"q": s["q_out"], "k": s["k_out"]} if rotate else {}
    if s["case"]["kv"] == "fp4":
        P.puzzle_kv_read_tokens(s["desc"], s["view"], s["k_read"], s["v_read"], read_lens=s["read_lens"])
        return dict(out, k_read=s["k_read"], v_read=s["v_read"])
    return dict(out, k_cache=_as_values(s["k_cache"]), v_cache=_as_values(s["v_cache"]))


def _as_values(cache):
    return cache.view(torch.float8_e4m3fn) if cache.dtype == torch.uint8 else cache


def _plain_attention(s, b, q, k, v, scale, out, lse):
    """Sequence b: q float32 [n][64][64] at the last n of the m keys k, v float32 [m][8][64]; writes its rows of out, lse."""
    n, m, window = q.shape[0], k.shape[0], s["case"]["window"]
    kt, vt = k.permute(1, 2, 0), v.transpose(0, 1)                              # [8][64][m], [8][m][64]
    t = torch.arange(m, device="cuda")
    sink = s["sinks"].view(HKV, GROUP, 1)
    step = max(1, (1 << 28) // (HQ * m))
    for i0 in range(0, n, step):
        x = q[i0:i0 + step].view(-1, HKV, GROUP, D).permute(1, 2, 0, 3)        # [8][8][rows][64]
        rows = x.shape[2]
        logit = torch.matmul(x.reshape(HKV, GROUP * rows, D) * scale, kt).view(HKV, GROUP, rows, m)
        p = (m - n + i0 + torch.arange(rows, device="cuda"))[:, None]
        hidden = t > p
        if window:
            hidden = hidden | (t <= p - window)
        logit.masked_fill_(hidden, -math.inf)
        top = torch.maximum(logit.amax(-1), sink)
        w = logit.sub_(top[..., None]).exp_()
        z = w.sum(-1) + torch.exp(sink - top)
        o = torch.matmul(w.view(HKV, GROUP * rows, m), vt).view(HKV, GROUP, rows, D) / z[..., None]
        at = s["first"][b] + i0
        out[at:at + rows] = o.permute(2, 0, 1, 3).reshape(rows, HQ, D).bfloat16()
        lse[at:at + rows] = (top + torch.log(z)).permute(2, 0, 1).reshape(rows, HQ)


def _plain_prompt(s):
    out, lse = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    for b, n in enumerate(s["new"]):
        if n:
            x = s["qkv"][s["first"][b]:s["first"][b] + n].float()
            _plain_attention(s, b, x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], D ** -0.5, out, lse)
    return {"out": out, "lse": lse}


def _logical(s, name, b, lo, hi):
    """Tokens [lo, hi) of sequence b, float32 [hi - lo][8][64]."""
    first = lo // BLOCK
    x = s[name + "_cache"][s["table"][b, first:-(-hi // BLOCK)].long()]
    kv = s["case"]["kv"]
    x = _dequantise4(*_unpack4(x, name == "v")) if kv == "fp4" else _as_values(x).float()
    x = x.transpose(1, 2).flatten(0, 1)[lo - first * BLOCK:hi - first * BLOCK]
    return x if kv == "bf16" else x * s[name + "_scale"][:, None]


def _plain_chunk(s):
    out, lse = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    window = s["case"]["window"]
    for b, n in enumerate(s["new"]):
        if n:
            m = s["context"][b]
            lo = max(0, m - n + 1 - window) if window else 0                   # keys before it are seen by none
            q = s["q"][s["first"][b]:s["first"][b] + n].float()
            _plain_attention(s, b, q, _logical(s, "k", b, lo, m), _logical(s, "v", b, lo, m), D ** -0.5, out, lse)
    return {"out": out, "lse": lse}


def _places(s):
    """Of every packed token: its sequence and its position."""
    new = torch.tensor(s["new"])
    seq = torch.repeat_interleave(torch.arange(len(s["new"])), new)
    pos = torch.arange(len(seq)) - torch.tensor(s["first"][:-1])[seq] + (torch.tensor(s["context"]) - new)[seq]
    return seq.cuda(), pos.cuda()


def _plain_append(s):
    case = s["case"]
    kv, r = case["kv"], case["rotary"]
    seq, pos = _places(s)
    x = s["qkv"].float()
    out = {}
    if case["rotate"]:
        rows = s["cos_sin"][pos][:, None]
        cos, sin = rows[..., :r // 2], rows[..., r // 2:]
        turn, rest = x[:, :HQ + HKV, :r], x[:, :HQ + HKV, r:]
        if case["interleaved"]:
            a, b = turn[..., 0::2], turn[..., 1::2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = turn[..., :r // 2], turn[..., r // 2:]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        turned = torch.cat([turned, rest], -1)
        out = {"q": turned[:, :HQ].bfloat16(), "k": turned[:, HQ:].bfloat16()}
    else:
        turned = x[:, :HQ + HKV]
    block, slot = s["table"].long()[seq, pos // BLOCK], pos % BLOCK
    inside = pos - (torch.tensor(s["context"]) - torch.tensor(s["new"])).cuda()[seq]
    for name, y in (("k", turned[:, HQ:]), ("v", x[:, HQ + HKV:])):
        scale = s[name + "_scale"][:, None]
        if kv == "fp4":
            read = torch.zeros(len(s["new"]), max(s["new"]), HKV, D, dtype=torch.bfloat16, device="cuda")
            read[seq, inside] = (_dequantise4(*_quantise4(y / scale)) * scale).bfloat16()
            out[name + "_read"] = read
        else:
            cache = s[name + "_cache"]
            cache[block, :, slot] = y.bfloat16() if kv == "bf16" else _e4m3(y / scale).view(torch.uint8)
            out[name + "_cache"] = _as_values(cache)
    return out


# -------------------------------------------------------------------------------------------------------- work ----

def work(case):
    new, context = _lens(case)
    total, window = sum(new), case.get("window", 0)
    value = {"fp8": 1.0, "bf16": 2.0, "fp4": 0.5625}[case.get("kv", "bf16")]
    if case["op"] != "append":
        pairs = keys = 0
        for n, m in zip(new, context):
            if not n:
                continue
            lo = max(0, m - n + 1 - window) if window else 0
            keys += m - lo
            if window:
                grow = max(0, min(n, window - (m - n)))                        # tokens that do not fill the window yet
                pairs += grow * (m - n) + grow * (grow + 1) // 2 + (n - grow) * window
            else:
                pairs += n * (m - n) + n * (n + 1) // 2
        return {"bytes": keys * HKV * 2 * D * value + total * HQ * (4 * D + 4), "flops": pairs * HQ * 4 * D}
    kv = 2 * total * HKV * D
    moved = kv * (2 + value) + (kv * 2 if case["kv"] == "fp4" else 0)
    flops = 6.0 * kv
    if case["rotate"]:
        moved += total * (4 * HQ * D + 2 * HKV * D + 4 * case["rotary"])
        flops += 3 * total * (HQ + HKV) * case["rotary"]
    return {"bytes": moved, "flops": flops}


# ------------------------------------------------------------------------------------------------------- exact ----

def _near(y, lowest, bits, most):
    """y rounded to `bits` fraction bits, ties to even, exponents from `lowest` on, at most `most`, in 64 bits."""
    e = torch.frexp(y)[1] - 1
    step = torch.ldexp(torch.ones_like(y), e.clamp(min=lowest) - bits)
    return (torch.round(y / step) * step).clamp(-most, most)


def _stand4(y):
    """What the 4-bit cache keeps of y [..., 64], in 64 bits."""
    g = y.reshape(*y.shape[:-1], 4, 16)
    t = _near(g.abs().amax(-1, keepdim=True) / 6, -6, 3, 448.0)
    return torch.where(t > 0, _near(g / t.clamp(min=2.0 ** -9), 0, 1, 6.0) * t, torch.zeros_like(g)).reshape(y.shape)


def _cached(s, name, b, lo, hi):
    """Tokens [lo, hi) of sequence b, float64 [hi - lo][8][64], from the cache's bytes; the head's scale included."""
    t = torch.arange(lo, hi, device="cuda")
    block = s["table"][b].long()[t // BLOCK]
    t = (t % BLOCK)[:, None]
    cache = s[name + "_cache"]
    if cache.dtype == torch.bfloat16:
        return cache[block, :, t[:, 0]].double()
    scale = s[name + "_scale"].double()[:, None]
    if cache.dim() == 4:
        return cache[block, :, t[:, 0]].view(torch.float8_e4m3fn).double() * scale
    d = torch.arange(D, device="cuda")
    if name == "k":
        byte, odd, at = 32 * t + d // 2, (d % 2).expand(len(t), D), 16 * (d // 16) + 2 * (t % 8) + t // 8
    else:
        byte, odd = 256 * (d // 32) + 32 * (t // 2) + d % 32, (t % 2).expand(len(t), D)
        at = 16 * (d // 16) + 4 * (t % 8 // 2) + 2 * (t // 8) + t % 2
    rows = cache[block].transpose(0, 1)                                         # [8][tokens][576]
    code = rows.gather(2, byte.expand(HKV, -1, -1)).int() >> (4 * odd) & 15
    exponent, fraction = (code >> 1 & 3).double(), (code & 1).double()
    size = torch.where(exponent > 0, (1 + fraction / 2) * torch.exp2(exponent - 1), fraction / 2)
    block_scale = rows.gather(2, (512 + at).expand(HKV, -1, -1)).view(torch.float8_e4m3fn).double()
    value = torch.where(code >= 8, -size, size) * block_scale
    return value.transpose(0, 1) * scale


def exact(case, seed):
    s = prepare(case, seed)
    new, context, first = s["new"], s["context"], s["first"]
    total = first[-1]
    if case["op"] != "append":
        window = case["window"]
        out = torch.zeros(total, HQ, D, dtype=torch.float64, device="cuda")
        lse = torch.zeros(total, HQ, dtype=torch.float64, device="cuda")
        for b, n in enumerate(new):
            m = context[b]
            for i0 in range(0, n, 512):                                        # the keys these queries can see at all
                i1 = min(n, i0 + 512)
                hi = m - n + i1
                lo = max(0, m - n + i0 + 1 - window) if window else 0
                if case["op"] == "prompt":
                    rows = s["qkv"][first[b] + lo:first[b] + hi]
                    k, v = rows[:, HQ:HQ + HKV].double(), rows[:, HQ + HKV:].double()
                else:
                    k, v = _cached(s, "k", b, lo, hi), _cached(s, "v", b, lo, hi)
                p = torch.arange(m - n + i0, hi, device="cuda")[:, None]
                j = torch.arange(lo, hi, device="cuda")[None]
                seen = j <= p
                if window:
                    seen &= j + window > p
                bias = torch.where(seen, 0.0, -math.inf).double()
                for h in range(HQ):
                    q = s["q"][first[b] + i0:first[b] + i1, h].double()
                    x = torch.addmm(bias, q, k[:, h // GROUP].T, alpha=1 / math.sqrt(D))
                    whole = torch.logaddexp(torch.logsumexp(x, -1), s["sinks"][h].double())
                    lse[first[b] + i0:first[b] + i1, h] = whole
                    out[first[b] + i0:first[b] + i1, h] = torch.exp(x - whole[:, None]) @ v[:, h // GROUP]
        return {"out": out, "lse": lse}
    kv, r = case["kv"], case["rotary"]
    x = s["qkv"].double()
    out = {}
    if kv == "fp4":
        for name in ("k_read", "v_read"):
            out[name] = torch.zeros(len(new), max(new), HKV, D, dtype=torch.float64, device="cuda")
    else:
        out = {"k_cache": _as_values(s["k_cache"]).double(), "v_cache": _as_values(s["v_cache"]).double()}
    for b, n in enumerate(new):
        if not n:
            continue
        rows = x[first[b]:first[b] + n]
        pos = torch.arange(context[b] - n, context[b], device="cuda")
        if case["rotate"]:
            row = s["cos_sin"][pos].double()
            turn = torch.complex(row[:, :r // 2], row[:, r // 2:])[:, None]
            part = rows[:, :HQ + HKV, :r].clone()
            if case["interleaved"]:
                z = torch.view_as_complex(part.unflatten(-1, (r // 2, 2)).contiguous()) * turn
                part = torch.view_as_real(z).flatten(-2)
            else:
                z = torch.complex(part[..., :r // 2].contiguous(), part[..., r // 2:].contiguous()) * turn
                part = torch.cat([z.real, z.imag], -1)
            rows[:, :HQ + HKV, :r] = part
        where = s["table"][b].long()[pos // BLOCK], pos % BLOCK
        for name, y in (("k", rows[:, HQ:HQ + HKV]), ("v", rows[:, HQ + HKV:])):
            scale = s[name + "_scale"].double()[:, None]
            if kv == "fp4":
                out[name + "_read"][b, :n] = _stand4(y / scale) * scale
            else:
                out[name + "_cache"][where[0], :, where[1]] = y if kv == "bf16" else _near(y / scale, -6, 3, 448.0)
    if case["rotate"]:
        out["q"], out["k"] = x[:, :HQ], x[:, HQ:HQ + HKV]
    return out
