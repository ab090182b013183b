"""Operators around the 4-bit key/value cache, as they are measured: position rotation with quantise-and-append,
reading cached tokens back, and decode attention over a cache of E2M1 codes.

`run` with `own` false computes the plain forms in elementary torch operations; with `own` true it makes the calls a
user of the package makes.  All caches are paged in blocks of 16 tokens, 64 query heads on 8 KV heads of 64 channels.

4-bit cache, one (block, KV head) = 576 bytes: 512 bytes of E2M1 codes, then 64 E4M3 scales, one per token and 16
channels.  K codes: token t at bytes 32 t .. 32 t + 31, channel d in byte d / 2 (even channel in the low nibble).
V codes: byte 256 (d / 32) + 32 (t / 2) + d % 32 (even token in the low nibble).  With b = d / 16, the scale of K is
byte 16 b + 2 (t % 8) + t / 8 of the 64, that of V byte 16 b + 4 ((t % 8) / 2) + 2 (t / 8) + t % 2.
"""
import math

import torch

own = False

HQ, HKV, D, BLOCK = 64, 8, 64, 16
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------------------------------- cases ----

def listed():
    append = dict(op="append", interleaved=False, rotary=64, ragged=False, far=False)
    attn = dict(n_q=1, window=0, ragged=False, paged=True)
    return [
        # one decode step's new token for a small batch into the E4M3 cache: nothing but latency
        dict(append, name="step_fp8_b16", kv="fp8", batch=16, n_new=1, context=2048),
        # the same for a serving batch into the 4-bit cache; the rounded token is read back
        dict(append, name="step_fp4_b64", kv="fp4", batch=64, n_new=1, context=2048, far=True),
        # a prompt chunk of 2048 tokens for 16 sequences
        dict(append, name="chunk_fp8_16x2048", kv="fp8", batch=16, n_new=2048, context=2048),
        # ragged odd chunks into the bf16 cache, adjacent pairs rotated, half of the channels only
        dict(append, name="chunk_bf16_5x777", kv="bf16", batch=5, n_new=777, context=2500, interleaved=True, rotary=32,
             ragged=True),
        # a prompt chunk into the 4-bit cache, read back so that the chunk's own attention sees the rounded values
        dict(append, name="chunk_fp4_8x1000", kv="fp4", batch=8, n_new=1000, context=4100, ragged=True, far=True),
        # a whole 4-bit cache read back as bf16: moving sequences to another worker
        dict(name="read_fp4_16x8192", op="read", kv="fp4", batch=16, n_new=8192, context=8192, ragged=False),
        # a small batch at a short context: latency
        dict(attn, name="decode_fp4_b4_1k", op="decode", batch=4, context=1024, paged=False),
        # a layer with a 128-token window
        dict(attn, name="decode_fp4_b32_w128", op="decode", batch=32, context=8192, window=128),
        # the long-context step: 16 sequences of 64K tokens
        dict(attn, name="decode_fp4_b16_64k", op="decode", batch=16, context=65536),
        # ragged long contexts, odd lengths
        dict(attn, name="decode_fp4_b24_ragged", op="decode", batch=24, context=40001, ragged=True),
        # two tokens per sequence (a drafted token verified) at 64K
        dict(attn, name="tokens2_fp4_b16_64k", op="decode", batch=16, context=65536, n_q=2),
        # five drafted tokens, ragged, on a layer with a 500-token window
        dict(attn, name="tokens5_fp4_b7_w500", op="decode", batch=7, context=9001, window=500, n_q=5, ragged=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "append", "read", "decode", "decode", "decode"))
    if op == "decode":
        n_q = rng.choice((1, 1, 1, 2, 3, 4, 6))
        context = _log(rng, 16, 65536)
        batch = _log(rng, 1, max(1, min(64, (1 << 20) // (n_q * context))))
        window = rng.choice((0, 0, 0, 128, _log(rng, 1, 8192)))
        return dict(op=op, batch=batch, context=context, n_q=n_q, window=window, ragged=rng.random() < 0.5,
                    paged=rng.random() < 0.8)
    kv = rng.choice(("fp8", "fp4", "fp4", "bf16"))
    n_new = _log(rng, 1, 4096)
    batch = _log(rng, 1, max(1, min(64, 32768 // n_new)))
    context = n_new + rng.randrange(0, 2048)
    if op == "read":
        return dict(op=op, kv=kv, batch=batch, n_new=n_new, context=context, ragged=rng.random() < 0.5)
    return dict(op=op, kv=kv, batch=batch, n_new=n_new, context=context, interleaved=rng.random() < 0.3,
                rotary=rng.choice((64, 64, 32, 48)), ragged=rng.random() < 0.5, far=rng.random() < 0.3)


# -------------------------------------------------------------------------------------------------- 4-bit format ----

def _e4m3(x):
    """Float32 to the nearest E4M3 value, ties to even, saturating; the codes' bytes."""
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
    shape, parts = (BLOCK, D), []
    for lo in range(0, nb, 8192):
        x = torch.randn((min(8192, nb - lo), HKV) + shape, generator=_gen(seed, k + 100 + lo), device="cuda")
        y = x / scale[None, :, None, None]
        if kv == "fp4":
            parts.append(_pack4(*_quantise4(y), is_v))
        else:
            parts.append(x.bfloat16() if kv == "bf16" else _e4m3(y).view(torch.uint8))
    return torch.cat(parts)


def prepare(case, seed):
    batch, context = case["batch"], case["context"]
    kv = case.get("kv", "fp4")
    per_seq = -(-context // BLOCK)
    nb = batch * per_seq
    g = _gen(seed, 1)
    lens = torch.full((batch,), context, dtype=torch.int32, device="cuda")
    if case["ragged"]:
        lens = torch.randint(max(1, context // 3), context + 1, (batch,), generator=g, device="cuda", dtype=torch.int32)
    table = None
    if case.get("paged", True):
        table = torch.randperm(nb, generator=g, device="cuda").to(torch.int32).view(batch, per_seq)
    # scales as a max calibration of N(0, 1) samples leaves them: about amax / 448, another for each head
    s = {"case": case, "lens": lens, "table": table, "per_seq": per_seq}
    for k, name in enumerate(("k", "v")):
        s[name + "_scale"] = (0.008 + 0.004 * torch.rand(HKV, generator=g, device="cuda"))
        s[name + "_cache"] = _fill(kv, nb, s[name + "_scale"], seed, 10 + k, k == 1)
    if case["op"] == "decode":
        n_q = case["n_q"]
        s["q"] = torch.randn(batch, n_q, HQ, D, generator=g, device="cuda").bfloat16()
        s["sinks"] = torch.randn(HQ, generator=g, device="cuda")
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(batch, n_q, HQ, device="cuda")
    else:
        n = case["n_new"]
        s["new_lens"] = None
        if case["ragged"]:
            s["new_lens"] = torch.randint(0, n + 1, (batch,), generator=g, device="cuda", dtype=torch.int32)
        if case["op"] == "append":
            # q, k and v are slices of one projection's output
            s["qkv"] = torch.randn(batch, n, HQ + 2 * HKV, D, generator=g, device="cuda").bfloat16()
            s["offset"] = None
            if case["far"]:
                s["offset"] = torch.randint(0, 120000, (batch,), generator=g, device="cuda", dtype=torch.int32)
            r, m = case["rotary"], 131072
            angle = torch.arange(m, device="cuda", dtype=torch.float64)[:, None] * torch.pow(
                150000.0, -torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)
            s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], -1).float()
            s["q_out"] = torch.zeros(batch, n, HQ, D, dtype=torch.bfloat16, device="cuda")
        s["k_out"] = torch.zeros(batch, n, HKV, D, dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.zeros_like(s["k_out"])
    if own:  # the descriptors and the workspace, which a program makes once per layer
        _plan(s, kv)
    return s


def _plan(s, kv):
    import paper_2602_11937_b200 as P
    case = s["case"]
    s["desc"] = P.layer_desc(window=case.get("window", 0), kv_dtype={"fp8": P.KV_FP8_E4M3, "bf16": P.KV_BF16,
                                                                     "fp4": P.KV_FP4_E2M1}[kv])
    s["view"] = P.kv_view(s["k_cache"], s["v_cache"], s["lens"], block_table=s["table"],
                          max_blocks_per_seq=s["per_seq"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    if case["op"] == "decode":
        batch, n_q = case["batch"], case["n_q"]
        size, init = P.puzzle_decode_attn_workspace_bytes, P.puzzle_decode_attn_workspace_init
        shape = (s["desc"], batch)
        if n_q > 1:
            size, init = P.puzzle_decode_attn_tokens_workspace_bytes, P.puzzle_decode_attn_tokens_workspace_init
            shape += (n_q,)
        s["workspace"] = torch.empty(size(*shape), dtype=torch.uint8, device="cuda")
        init(*shape, s["workspace"])
    elif case["op"] == "append":
        s["rope"] = P.rope_view(s["cos_sin"], interleaved=case["interleaved"], pos_offset=s["offset"])


# --------------------------------------------------------------------------------------------------------- run ----

def run(s):
    op = s["case"]["op"]
    if own:
        return {"append": _own_append, "read": _own_read, "decode": _own_decode}[op](s)
    return {"append": _plain_append, "read": _plain_read, "decode": _plain_decode}[op](s)


def _own_append(s):
    import paper_2602_11937_b200 as P
    case, qkv = s["case"], s["qkv"]
    q, k, v = qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HKV], qkv[:, :, HQ + HKV:]
    P.puzzle_kv_append_rope(s["desc"], s["view"], s["rope"], q, k, v, s["q_out"], new_lens=s["new_lens"])
    if case["kv"] == "fp4":
        return dict(_own_read(s), q=s["q_out"])
    return {"q": s["q_out"], "k_cache": _as_values(s["k_cache"]), "v_cache": _as_values(s["v_cache"])}


def _own_read(s):
    import paper_2602_11937_b200 as P
    P.puzzle_kv_read_tokens(s["desc"], s["view"], s["k_out"], s["v_out"], read_lens=s["new_lens"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_decode(s):
    import paper_2602_11937_b200 as P
    if s["case"]["n_q"] > 1:
        P.puzzle_decode_attn_tokens(s["desc"], s["view"], s["q"], s["sinks"], s["out"], s["lse"],
                                    workspace=s["workspace"])
    else:
        P.puzzle_decode_attn(s["desc"], s["view"], s["q"][:, 0], s["sinks"], s["out"][:, 0], s["lse"][:, 0],
                             workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def _as_values(cache):
    return cache.view(torch.float8_e4m3fn) if cache.dtype == torch.uint8 else cache


def _rows(s, n):
    """Positions [batch][n] of the last tokens of every sequence, and which of them are real (the others are put at 0)."""
    count = s["new_lens"] if s.get("new_lens") is not None else torch.full_like(s["lens"], n)
    i = torch.arange(n, device="cuda")[None]
    pos = (s["lens"] - count)[:, None] + i
    real = (i < count[:, None]) & (pos >= 0)
    return torch.where(real, pos, torch.zeros_like(pos)), real


def _blocks(s, block):
    """Physical blocks of logical blocks [batch][m]."""
    if s["table"] is None:
        return block + (torch.arange(block.shape[0], device="cuda") * s["per_seq"])[:, None]
    return s["table"].long().gather(1, block)


def _plain_append(s):
    case = s["case"]
    n, r, kv = case["n_new"], case["rotary"], case["kv"]
    pos, real = _rows(s, n)
    at = pos if s["offset"] is None else pos + s["offset"][:, None]
    rows = s["cos_sin"][at][:, :, None]
    cos, sin = rows[..., :r // 2], rows[..., r // 2:]
    x = s["qkv"].float()
    turn, rest = x[:, :, :HQ + HKV, :r], x[:, :, :HQ + HKV, r:]
    if case["interleaved"]:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turn[..., :r // 2], turn[..., r // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    turned = torch.cat([turned, rest], -1)
    out = {"q": torch.where(real[:, :, None, None], turned[:, :, :HQ], torch.zeros_like(turned[:, :, :HQ])).bfloat16()}
    pick = (lambda y: y.flatten(0, 1)) if s["new_lens"] is None else (lambda y: y[real])
    blk, slot = pick(_blocks(s, pos // BLOCK)), pick(pos % BLOCK)
    for name, y in (("k", turned[:, :, HQ:]), ("v", x[:, :, HQ + HKV:])):
        scale = s[name + "_scale"][:, None]
        if kv == "fp4":
            value = _dequantise4(*_quantise4(y / scale)) * scale
            out[name] = torch.where(real[:, :, None, None], value, torch.zeros_like(value)).bfloat16()
        else:
            cache = s[name + "_cache"]
            cache[blk, :, slot] = pick(y.bfloat16() if kv == "bf16" else _e4m3(y / scale).view(torch.uint8))
            out[name + "_cache"] = _as_values(cache)
    return out


def _logical(s, name, kv, nblk):
    """The first nblk blocks of every sequence, float32 [batch][16 nblk][Hkv][64] in units of the head's scale."""
    index = torch.arange(nblk, device="cuda").expand(s["lens"].shape[0], nblk)
    x = s[name + "_cache"][_blocks(s, index)]
    if kv == "fp4":
        x = _dequantise4(*_unpack4(x, name == "v"))
    else:
        x = _as_values(x).float()
    return x.permute(0, 1, 3, 2, 4).flatten(1, 2)


def _plain_read(s):
    case = s["case"]
    pos, real = _rows(s, case["n_new"])
    out = {}
    for name in ("k", "v"):
        x = _logical(s, name, case["kv"], s["per_seq"])
        x = x.gather(1, pos[:, :, None, None].expand(-1, -1, HKV, D))
        if case["kv"] != "bf16":
            x = x * s[name + "_scale"][:, None]
        out[name] = torch.where(real[:, :, None, None], x, torch.zeros_like(x)).bfloat16()
    return out


def _plain_decode(s):
    case = s["case"]
    n_q, window = case["n_q"], case["window"]
    batch = case["batch"]
    k = _logical(s, "k", "fp4", s["per_seq"])
    v = _logical(s, "v", "fp4", s["per_seq"])
    q = s["q"].float().view(batch, n_q, HKV, HQ // HKV, D) * (s["k_scale"] / math.sqrt(D))[:, None, None]
    logit = torch.einsum("bqhgd,bthd->bqhgt", q, k).flatten(2, 3)
    end = (s["lens"][:, None] - n_q + torch.arange(n_q, device="cuda"))[:, :, None, None]     # the token's own position
    t = torch.arange(k.shape[1], device="cuda")
    seen = t <= end
    if window:
        seen = seen & (t > end - window)
    logit = torch.where(seen, logit, torch.full_like(logit, -math.inf))
    sink = s["sinks"].expand(batch, n_q, HQ)
    top = torch.maximum(logit.amax(-1), sink)
    w = torch.exp(logit - top[..., None])
    z = w.sum(-1) + torch.exp(sink - top)
    o = torch.einsum("bqhgt,bthd->bqhgd", w.view(batch, n_q, HKV, HQ // HKV, -1), v) * s["v_scale"][:, None, None]
    return {"out": (o.flatten(2, 3) / z[..., None]).bfloat16(), "lse": top + torch.log(z)}


# -------------------------------------------------------------------------------------------------------- work ----

def work(case):
    """Every sequence counted at its mean length where lengths are drawn."""
    batch, context = case["batch"], case["context"]
    value = {"fp8": 1.0, "bf16": 2.0, "fp4": 0.5625}[case.get("kv", "fp4")]
    if case["op"] == "decode":
        n_q, window = case["n_q"], case["window"]
        mean = context * 2 / 3 if case["ragged"] else context
        seen = min(mean, window + n_q - 1) if window else mean
        own_keys = min(mean, window) if window else mean
        return {"bytes": batch * (seen * HKV * 2 * D * value + n_q * HQ * (4 * D + 4)),
                "flops": batch * n_q * own_keys * HQ * 4 * D}
    n = case["n_new"] * (0.5 if case["ragged"] else 1.0)
    kv = 2 * batch * n * HKV * D
    if case["op"] == "read":
        return {"bytes": kv * (value + 2), "flops": 2 * kv}
    q = batch * n * HQ * D
    back = kv * 2 if case["kv"] == "fp4" else 0
    return {"bytes": 4 * q + kv * (2 + value) + batch * n * 4 * case["rotary"] + back,
            "flops": 3 * q * case["rotary"] / D + 6 * kv}


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
    """Tokens [lo, hi) of sequence b, float64 [hi - lo][Hkv][64], from the cache's bytes; the head's scale included."""
    t = torch.arange(lo, hi, device="cuda")
    block = t // BLOCK
    block = s["table"][b].long()[block] if s["table"] is not None else block + b * s["per_seq"]
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
    rows = cache[block].transpose(0, 1)                                         # [Hkv][tokens][576]
    code = rows.gather(2, byte.expand(HKV, -1, -1)).int() >> (4 * odd) & 15
    exponent, fraction = (code >> 1 & 3).double(), (code & 1).double()
    size = torch.where(exponent > 0, (1 + fraction / 2) * torch.exp2(exponent - 1), fraction / 2)
    block_scale = rows.gather(2, (512 + at).expand(HKV, -1, -1)).view(torch.float8_e4m3fn).double()
    value = torch.where(code >= 8, -size, size) * block_scale
    return value.transpose(0, 1) * scale


def exact(case, seed):
    s = prepare(case, seed)
    batch = case["batch"]
    lens = s["lens"].tolist()
    if case["op"] == "decode":
        n_q, window = case["n_q"], case["window"]
        out = torch.zeros(batch, n_q, HQ, D, dtype=torch.float64, device="cuda")
        lse = torch.zeros(batch, n_q, HQ, dtype=torch.float64, device="cuda")
        sink = s["sinks"].double()[:, None]
        for b in range(batch):
            first = max(0, lens[b] - n_q + 1 - window) if window else 0
            k, v = (_cached(s, name, b, first, lens[b]).transpose(0, 1) for name in ("k", "v"))      # [Hkv][t][64]
            for i in range(n_q):
                end = lens[b] - n_q + i + 1
                if end <= 0:
                    lse[b, i] = sink[:, 0]
                    continue
                lo = max(0, end - window) - first if window else 0
                q = s["q"][b, i].double().view(HKV, HQ // HKV, D)
                x = (q @ k[:, lo:end - first].transpose(1, 2) / math.sqrt(D)).view(HQ, -1)
                x = torch.cat([x, sink], -1)
                lse[b, i] = torch.logsumexp(x, -1)
                w = torch.exp(x[:, :-1] - lse[b, i][:, None]).view(HKV, HQ // HKV, -1)
                out[b, i] = (w @ v[:, lo:end - first]).view(HQ, D)
        return {"out": out, "lse": lse}
    n = case["n_new"]
    counts = s["new_lens"].tolist() if s["new_lens"] is not None else [n] * batch
    if case["op"] == "read":
        out = {name: torch.zeros(batch, n, HKV, D, dtype=torch.float64, device="cuda") for name in ("k", "v")}
        for b in range(batch):
            skip = max(0, counts[b] - lens[b])
            for name in out:
                out[name][b, skip:counts[b]] = _cached(s, name, b, lens[b] - counts[b] + skip, lens[b])
        return out
    kv, r = case["kv"], case["rotary"]
    q = torch.zeros(batch, n, HQ, D, dtype=torch.float64, device="cuda")
    if kv == "fp4":
        out = {"q": q, "k": torch.zeros(batch, n, HKV, D, dtype=torch.float64, device="cuda")}
        out["v"] = torch.zeros_like(out["k"])
    else:
        out = {"q": q, "k_cache": _as_values(s["k_cache"]).double(), "v_cache": _as_values(s["v_cache"]).double()}
    for b in range(batch):
        skip = max(0, counts[b] - lens[b])
        i = torch.arange(skip, counts[b], device="cuda")
        pos = lens[b] - counts[b] + i
        row = s["cos_sin"][pos + (int(s["offset"][b]) if s["offset"] is not None else 0)].double()
        turn = torch.complex(row[:, :r // 2], row[:, r // 2:])[:, None]
        x = s["qkv"][b, i].double()
        part = x[:, :HQ + HKV, :r].clone()
        if case["interleaved"]:
            z = torch.view_as_complex(part.unflatten(-1, (r // 2, 2)).contiguous()) * turn
            part = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(part[..., :r // 2].contiguous(), part[..., r // 2:].contiguous()) * turn
            part = torch.cat([z.real, z.imag], -1)
        x[:, :HQ + HKV, :r] = part
        q[b, i] = x[:, :HQ]
        where = s["table"][b].long()[pos // BLOCK], pos % BLOCK
        for name, y in (("k", x[:, HQ:HQ + HKV]), ("v", x[:, HQ + HKV:])):
            scale = s[name + "_scale"].double()[:, None]
            if kv == "fp4":
                out[name][b, i] = _stand4(y / scale) * scale
            else:
                out[name + "_cache"][where[0], :, where[1]] = y if kv == "bf16" else _near(y / scale, -6, 3, 448.0)
    return out
