"""Plain references of the position rotation, the 4-bit format and the append / read-back of new tokens (numpy, one
value at a time where it matters).  Nothing here comes from the CUDA path; E4M3 codes come from the oracle's codec."""
from __future__ import annotations

import numpy as np

import oracle
from helpers import bf16_bits_to_f64

FP8, BF16, FP4 = oracle.KV_FP8_E4M3, oracle.KV_BF16, oracle.KV_FP4_E2M1
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([oracle.e4m3_decode(c) for c in range(256)])


def k_code_at(t, d):
    return 32 * t + d // 2, d % 2            # byte, nibble


def v_code_at(t, d):
    return 256 * (d // 32) + 32 * (t // 2) + d % 32, t % 2


def k_scale_at(t, b):
    return 512 + 16 * b + 2 * (t % 8) + t // 8


def v_scale_at(t, b):
    return 512 + 16 * b + 4 * ((t % 8) // 2) + 2 * (t // 8) + t % 2


def round_bf16(x):
    """float32 array -> bf16 bit patterns, nearest even; NaN -> 0x7FFF."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FFF), r)


def e2m1_encode(q):
    """Nearest E2M1 code of one float64 value: smallest distance, ties to the even code, saturating; sign kept."""
    a = abs(float(q))
    d = np.abs(E2M1 - min(a, 6.0))
    best = [c for c in range(8) if d[c] == d.min()]
    c = best[0] if len(best) == 1 else [c for c in best if c % 2 == 0][0]
    return c | (8 if np.signbit(q) else 0)


def fp4_quantise(y):
    """y float32 [64] -> codes [64], scale codes [4]."""
    codes, scales = np.zeros(64, np.uint8), np.zeros(4, np.uint8)
    for b in range(4):
        g = y[16 * b:16 * b + 16]
        if np.isnan(g).any():
            scales[b] = 0x7F
            continue
        with np.errstate(over="ignore"):
            scales[b] = oracle.e4m3_encode(np.float32(np.float32(np.abs(g).max()) / np.float32(6.0)))
        t = E4M3[scales[b]]
        if t == 0:
            continue
        for i in range(16):
            codes[16 * b + i] = e2m1_encode(np.float64(g[i]) / t)
    return codes, scales


def rotate(x_bits, cos_sin, pos, rotary, adjacent):
    """bf16 bits [H][64] of one token -> float32 [H][64] after the rotation; each product and sum rounded to float32."""
    x = bf16_bits_to_f64(x_bits).astype(np.float32)
    out = x.copy()
    half = rotary // 2
    c, s = cos_sin[pos, :half], cos_sin[pos, half:]
    i = np.arange(0, rotary, 2) if adjacent else np.arange(half)
    j = i + 1 if adjacent else i + half
    with np.errstate(invalid="ignore", over="ignore"):
        out[:, i] = x[:, i] * c - x[:, j] * s
        out[:, j] = x[:, j] * c + x[:, i] * s
    return out


class Cache:
    """One layer's cache as raw bytes (or bf16 bits) in the library's layout, with token-wise access."""

    def __init__(self, kind, nb, hkv, seed):
        r = np.random.default_rng(seed)
        self.kind, self.hkv = kind, hkv
        if kind == FP4:
            shape, hi, dt = (nb, hkv, 576), 256, np.uint8
        elif kind == FP8:
            shape, hi, dt = (nb, hkv, 16, 64), 256, np.uint8
        else:
            shape, hi, dt = (nb, hkv, 16, 64), 65536, np.uint16
        self.k, self.v = (r.integers(0, hi, size=shape).astype(dt) for _ in range(2))   # whatever was there before

    def put(self, blk, slot, h, is_v, x, x_bits, scale):
        """Writes float32 x [64] (for an unrotated bf16 row: x_bits) of one token."""
        c = (self.v if is_v else self.k)
        if self.kind == BF16:
            c[blk, h, slot] = x_bits if x_bits is not None else round_bf16(x)
            return
        with np.errstate(over="ignore", invalid="ignore"):
            y = (x / np.float32(scale)).astype(np.float32)
        if self.kind == FP8:
            c[blk, h, slot] = oracle.e4m3_encode_array(y)
            return
        codes, scales = fp4_quantise(y)
        p = c[blk, h]
        for d in range(64):
            byte, odd = v_code_at(slot, d) if is_v else k_code_at(slot, d)
            p[byte] = (p[byte] & (0x0F if odd else 0xF0)) | (codes[d] << (4 * odd))
        for b in range(4):
            p[v_scale_at(slot, b) if is_v else k_scale_at(slot, b)] = scales[b]

    def get(self, blk, slot, h, is_v):
        """float64 [64] of one token, the head's scale not applied."""
        c = (self.v if is_v else self.k)
        if self.kind == BF16:
            return bf16_bits_to_f64(c[blk, h, slot])
        if self.kind == FP8:
            return E4M3[c[blk, h, slot]]
        p, out = c[blk, h], np.zeros(64)
        for d in range(64):
            byte, odd = v_code_at(slot, d) if is_v else k_code_at(slot, d)
            t = E4M3[p[v_scale_at(slot, d // 16) if is_v else k_scale_at(slot, d // 16)]]
            out[d] = oracle.e2m1_decode(int(p[byte]) >> (4 * odd)) * t
        return out


def append(cache, table, max_blocks, seq_lens, new_lens, q, k, v, k_scale, v_scale, cos_sin=None, rotary=64,
           adjacent=False, offset=None):
    """Appends bf16-bit arrays [B][n][H][64] to `cache` in place; returns the rotated queries as bf16 bits, with the
    rows of skipped tokens left at 0xDEAD.  cos_sin None: no rotation."""
    B, n = k.shape[:2]
    nb = cache.k.shape[0]
    q_out = None if q is None else np.full(q.shape, 0xDEAD, dtype=np.uint16)
    for b in range(B):
        count = n if new_lens is None else min(max(int(new_lens[b]), 0), n)
        if seq_lens[b] <= 0 or seq_lens[b] > 16 * max_blocks:
            continue
        for i in range(count):
            pos = int(seq_lens[b]) - count + i
            if pos < 0:
                continue
            at = pos + (0 if offset is None else int(offset[b]))
            if cos_sin is not None and not 0 <= at < cos_sin.shape[0]:
                continue
            if q is not None and cos_sin is not None:
                q_out[b, i] = round_bf16(rotate(q[b, i], cos_sin, at, rotary, adjacent))
            blk = b * max_blocks + pos // 16 if table is None else int(table[b, pos // 16])
            if not 0 <= blk < nb:
                continue
            kr = bf16_bits_to_f64(k[b, i]).astype(np.float32) if cos_sin is None else \
                rotate(k[b, i], cos_sin, at, rotary, adjacent)
            vr = bf16_bits_to_f64(v[b, i]).astype(np.float32)
            for h in range(cache.hkv):
                cache.put(blk, pos % 16, h, False, kr[h], k[b, i, h] if cos_sin is None else None,
                          1.0 if k_scale is None else k_scale[h])
                cache.put(blk, pos % 16, h, True, vr[h], v[b, i, h], 1.0 if v_scale is None else v_scale[h])
    return q_out


def fp4_random_cache(nb, hkv, seed, scale=1.0):
    """K and V caches [nb][hkv][576] of N(0, scale) samples in 4 bits, quantised in whole arrays (input preparation)."""
    r = np.random.default_rng(seed)
    out = []
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    t_idx, d_idx, b_idx = np.arange(16), np.arange(64), np.arange(4)
    for is_v in (False, True):
        x = (r.standard_normal((nb, hkv, 16, 4, 16)) * scale).astype(np.float32)
        sc = oracle.e4m3_encode_array((np.abs(x).max(-1) / np.float32(6)).astype(np.float32))
        t = E4M3[sc]
        code = np.searchsorted(borders, np.abs(x) / np.where(t > 0, t, 1.0)[..., None]).astype(np.uint8)
        code = np.where(t[..., None] > 0, code | (np.signbit(x).astype(np.uint8) << 3), 0).astype(np.uint8)
        code = code.reshape(nb, hkv, 16, 64)
        c = np.zeros((nb, hkv, 576), dtype=np.uint8)
        byte, odd = (v_code_at if is_v else k_code_at)(t_idx[:, None], d_idx[None, :])
        byte, odd = np.broadcast_arrays(byte, odd)
        for nib in (0, 1):
            m = odd == nib
            c[:, :, byte[m]] |= code[:, :, m] << (4 * nib)
        at = (v_scale_at if is_v else k_scale_at)(t_idx[:, None], b_idx[None, :])
        c[:, :, at] = sc
        out.append(c)
    return out
