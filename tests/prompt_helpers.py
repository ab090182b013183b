"""Plain 64-bit attention of packed tokens, caches of every type with a decoder of their bytes, and the tolerances of the
kernels' roundings.  Nothing here comes from the CUDA library."""
from __future__ import annotations

import math

import torch

import paper_2602_11937_b200 as P

D, BLOCK = 64, 16
KINDS = {"fp8": P.KV_FP8_E4M3, "bf16": P.KV_BF16, "fp4": P.KV_FP4_E2M1}
# half a step of the type that softmax weights are rounded to
WEIGHT = {"packed": 2.0 ** -8, "bf16": 2.0 ** -8, "fp8": 2.0 ** -11, "fp4": 2.0 ** -11}
# An f16 weight lies at 2^9 of its value in units of the reference, which is less than twice the row's largest weight: half a step
# of f16's smallest numbers, 2^-25, is 2^-33 of the largest weight, and a second rounding, where the reference moved between the
# halves of 64 keys, half of that.  So much each of the keys that a row sees can add or lose: 1.5 x 2^-33 < 2^-32.
FLOOR = {"packed": 0.0, "bf16": 0.0, "fp8": 2.0 ** -32, "fp4": 2.0 ** -32}
SLOP = 2.0 ** -13      # float32 dot products of 64 terms, exponentials of arguments up to 2^5, sums: well inside


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make_starts(new, first=0):
    s = [first]
    for n in new:
        s.append(s[-1] + n)
    return s, torch.tensor(s, dtype=torch.int32, device="cuda")


def make_cache(kv, num_blocks, hkv, g):
    """Random bytes of a cache: K and V."""
    out = []
    for _ in range(2):
        if kv == "bf16":
            out.append(torch.randn(num_blocks, hkv, BLOCK, D, generator=g, device="cuda").bfloat16())
        elif kv == "fp8":
            x = torch.randn(num_blocks, hkv, BLOCK, D, generator=g, device="cuda") * 60
            out.append(x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
        else:
            c = torch.randint(0, 256, (num_blocks, hkv, 576), generator=g, device="cuda", dtype=torch.uint8)
            c[..., 512:] = torch.randint(0x48, 0x5c, (num_blocks, hkv, 64), generator=g, device="cuda", dtype=torch.uint8)
            out.append(c)
    return out


def cached(kv, cache, scale, blocks, lo, hi, is_v):
    """Tokens [lo, hi) of the sequence whose blocks are `blocks` (None entries: zeros), float64 [hi - lo][Hkv][64]."""
    t = torch.arange(lo, hi, device="cuda")
    block = blocks.long()[t // BLOCK]
    slot = t % BLOCK
    if kv == "bf16":
        return cache[block, :, slot].double()
    s = scale.double()[:, None]
    if kv == "fp8":
        return cache[block, :, slot].view(torch.float8_e4m3fn).double() * s
    d = torch.arange(D, device="cuda")
    tt = slot[:, None]
    if not is_v:
        byte, odd, at = 32 * tt + d // 2, (d % 2).expand(len(t), D), 16 * (d // 16) + 2 * (tt % 8) + tt // 8
    else:
        byte, odd = 256 * (d // 32) + 32 * (tt // 2) + d % 32, (tt % 2).expand(len(t), D)
        at = 16 * (d // 16) + 4 * (tt % 8 // 2) + 2 * (tt // 8) + tt % 2
    rows = cache[block].transpose(0, 1)
    hkv = cache.shape[1]
    code = rows.gather(2, byte.expand(hkv, -1, -1)).int() >> (4 * odd) & 15
    lut = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    size = lut[code & 7]
    block_scale = rows.gather(2, (512 + at).expand(hkv, -1, -1)).view(torch.float8_e4m3fn).double()
    return (torch.where(code >= 8, -size, size) * block_scale).transpose(0, 1) * s


def attention64(q, k, v, first, window, sinks, sm_scale, floor=0.0):
    """q [n][Hq][64] at positions first .. first + n - 1, keys [m][Hkv][64] at positions 0 ..; 64 bits.  Returns out, lse and
    the weighted sum of |v| that the roundings are relative to, with `floor` of each value on top."""
    n, hq, _ = q.shape
    m, hkv, _ = k.shape
    grp = hq // hkv
    out = torch.zeros(n, hq, D, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(out)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda")
    p = torch.arange(first, first + n, device="cuda")[:, None]
    j = torch.arange(m, device="cuda")[None]
    seen = j <= p
    if window:
        seen &= j > p - window
    for h in range(hq):
        kk, vv = k[:, h // grp], v[:, h // grp]
        x = (q[:, h].double() @ kk.T) * sm_scale
        x = torch.where(seen, x, torch.full_like(x, -math.inf))
        sink = sinks[h].double() if sinks is not None else torch.tensor(-math.inf, dtype=torch.float64, device="cuda")
        top = torch.maximum(x.amax(-1) if m else torch.full((n,), -math.inf, dtype=torch.float64, device="cuda"), sink)
        base = torch.where(torch.isinf(top) & (top < 0), torch.zeros_like(top), top)
        w = torch.where(seen, torch.exp(x - base[:, None]), torch.zeros_like(x))
        z = w.sum(-1) + torch.exp(sink - base)
        none = ~seen.any(-1)
        # a key that a row does not see is not in its sum, whatever its value is
        def mix(values):
            if torch.isfinite(values).all():
                return w @ values
            o = torch.zeros(n, D, dtype=torch.float64, device="cuda")
            for i in range(n):
                o[i] = w[i, seen[i]] @ values[seen[i]]
            return o
        zz = torch.where(none & (z == 0), torch.ones_like(z), z)[:, None]
        out[:, h] = mix(vv) / zz
        size[:, h] = mix(vv.abs()) / zz
        if floor:
            size[:, h] += floor / WEIGHT["fp8"] * (seen.double() @ torch.nan_to_num(vv.abs(), posinf=0.0))
        lse[:, h] = torch.where(z == 0, torch.full_like(z, -math.inf), base + torch.log(z))
    return out, lse, size


def check(what, got, lse, want, want_lse, size, weight):
    """Weights are off by `weight` of themselves, the output by half a bf16 step (2^-8) of itself."""
    got, lse = got.double(), lse.double()
    bound = (weight + SLOP) * size + 2.0 ** -8 * want.abs() + 1e-30
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got - want).abs() <= bound))
    assert not bad.any(), "%s: %d outputs off, worst %.3g of the bound, first at %s: %r, wanted %r" % (
        what, int(bad.sum()), float(((got - want).abs() / bound)[bad].max()), bad.nonzero()[0].tolist(),
        got[bad][0].item(), want[bad][0].item())
    same = (lse == want_lse) | (torch.isnan(lse) & torch.isnan(want_lse))
    bad = ~(same | ((lse - want_lse).abs() <= 2e-5 + 2.0 ** -19 * want_lse.abs()))
    assert not bad.any(), "%s: %d log sums off, first at %s: %r, wanted %r" % (
        what, int(bad.sum()), bad.nonzero()[0].tolist(), lse[bad][0].item(), want_lse[bad][0].item())
