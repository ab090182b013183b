"""CPU pins of the 4-bit format's reference: code values, layout, quantiser, attention; and the rotation table."""
import math

import numpy as np
import pytest
import torch

import oracle
from helpers import bf16_bits
import kv_reference as R


def test_code_values_and_signs():
    assert [oracle.e2m1_decode(c) for c in range(8)] == [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    for c in range(8):
        assert oracle.e2m1_decode(c | 8) == -oracle.e2m1_decode(c)


def test_layout_uses_every_nibble_and_scale_once():
    for code_at, scale_at in ((R.k_code_at, R.k_scale_at), (R.v_code_at, R.v_scale_at)):
        codes = {code_at(t, d) for t in range(16) for d in range(64)}
        assert codes == {(byte, nib) for byte in range(512) for nib in (0, 1)}
        assert sorted(scale_at(t, b) for t in range(16) for b in range(4)) == list(range(512, 576))


def test_encoder_takes_the_nearest_code_and_ties_go_to_even():
    for c in range(7):
        mid = (R.E2M1[c] + R.E2M1[c + 1]) / 2
        assert R.e2m1_encode(mid) == (c if c % 2 == 0 else c + 1)
        assert R.e2m1_encode(np.nextafter(mid, 0)) == c and R.e2m1_encode(np.nextafter(mid, 9)) == c + 1
    assert R.e2m1_encode(1e30) == 7 and R.e2m1_encode(-1e30) == 15 and R.e2m1_encode(-0.0) == 8


def test_quantiser_edges():
    codes, scales = R.fp4_quantise(np.zeros(64, np.float32))
    assert not codes.any() and not scales.any()
    y = np.ones(64, np.float32)
    y[3], y[20], y[40] = np.nan, np.inf, 1e9
    codes, scales = R.fp4_quantise(y)
    assert scales[0] == 0x7F and not codes[:16].any()                       # a group with a NaN reads as NaN
    assert scales[1] == 0x7E and codes[20] == 7 and not codes[21:32].any()  # saturates at 448 * 6
    assert scales[2] == 0x7E and codes[40] == 7 and R.E4M3[scales[3]] == 0.171875


def test_values_and_attention_agree_with_a_bf16_cache_of_the_same_values():
    """code * scale has at most six significant bits, so a bf16 cache holds the 4-bit cache's values exactly."""
    nb, hkv = 5, 2
    kc, vc = R.fp4_random_cache(nb, hkv, 3)
    c = R.Cache(R.FP4, nb, hkv, 0)
    c.k, c.v = kc, vc
    kd, vd = (np.stack([[[c.get(b, t, h, is_v) for t in range(16)] for h in range(hkv)] for b in range(nb)])
              for is_v in (False, True))
    as_bits = lambda x: bf16_bits(torch.from_numpy(x).to(torch.bfloat16))
    assert np.array_equal(torch.from_numpy(kd).to(torch.bfloat16).double().numpy(), kd)
    q = bf16_bits(torch.randn(1, 16, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16))
    table, lens = np.array([[4, 0, 2, 1, 3]], np.int32), np.array([71], np.int32)
    sinks = np.linspace(-1, 1, 16).astype(np.float32)
    for window in (0, 20):
        a, la = oracle.decode_attn(kc, vc, R.FP4, table, 5, lens, None, None, q, sinks, window, 0.125)
        b, lb = oracle.decode_attn(as_bits(kd), as_bits(vd), R.BF16, table, 5, lens, None, None, q, sinks, window, 0.125)
        assert np.array_equal(a, b) and np.array_equal(la, lb)
    # the head's scale multiplies the logits (K) and the output (V)
    ks, vs = np.array([0.5, 2.0], np.float32), np.array([4.0, 0.25], np.float32)
    a, _ = oracle.decode_attn(kc, vc, R.FP4, table, 5, lens, ks, vs, q, None, 0, 0.125)
    for h in range(2):
        rows = slice(8 * h, 8 * h + 8)
        b, _ = oracle.decode_attn(as_bits(kd), as_bits(vd), R.BF16, table, 5, lens, None, None, q, None, 0,
                                  0.125 * float(ks[h]))
        assert np.allclose(a[rows], b[rows] * vs[h], rtol=1e-13, atol=0)


def test_rope_table_rows_are_the_angles_of_their_position():
    import paper_2602_11937_b200 as P
    t = P.rope_table(120001, 32, theta=150000.0).double()
    assert t.shape == (120001, 32) and torch.all(t[0, :16] == 1) and torch.all(t[0, 16:] == 0)
    for p in (1, 777, 120000):
        for i in (0, 5, 15):
            a = p * 150000.0 ** (-2 * i / 32)
            assert abs(float(t[p, i]) - math.cos(a)) <= 2.0 ** -24 + 1e-10      # half a float32 step below 1
            assert abs(float(t[p, 16 + i]) - math.sin(a)) <= 2.0 ** -24 + 1e-10


def test_rope_table_stretched():
    import paper_2602_11937_b200 as P
    plain, long = P.rope_table(64, 64, theta=150000.0).double(), P.rope_table(64, 64, theta=150000.0, factor=32.0).double()
    gain = 0.1 * math.log(32.0) + 1.0
    assert torch.allclose(long[:, 0] / gain, plain[:, 0], atol=1e-6)            # the fastest frequency stays
    slow = 63 * 150000.0 ** (-62 / 64) / 32.0                                   # the slowest is divided by the factor
    assert abs(float(long[63, 63]) / gain - math.sin(slow)) < 1e-7
    for bad in (dict(num_positions=0), dict(num_positions=4, rotary_dim=3), dict(num_positions=4, factor=0.5)):
        with pytest.raises(ValueError):
            P.rope_table(**bad)
