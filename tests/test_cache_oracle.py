"""Pins of the compact cache's oracle (CPU): e4m3 rounding against torch's own
conversion, the rule of the scales, the rotation, the append's rules on blocks
with earlier tokens, and the window against a mask written out."""
import math

import numpy as np
import pytest
import torch

import cache_cases as C
from oracle import cache_oracle as CO


def test_codes_are_torchs():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(CO.TABLE, want)
    rng = np.random.default_rng(0)
    mids = (CO.TABLE[:126] + CO.TABLE[1:127]) / 2
    x = np.concatenate((CO.TABLE, mids, -mids, rng.standard_normal(4000) * 100, rng.standard_normal(4000) * 0.02)).astype(np.float32)
    x = x[~(np.abs(x) > 448)]
    got = CO.e4m3_code(x)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    nan = np.isnan(x)
    np.testing.assert_array_equal(got[~nan], want[~nan])
    assert np.isnan(CO.TABLE[got[nan]]).all()


@pytest.mark.parametrize("amax,e", [(0.0, -100), (448.0, 0), (449.0, 1), (447.9, 0), (1.75, -8), (1.7500001, -7), (1.0, -8),
                                    (3.3895e38, 120), (1e-45, -100), (2.0 ** -60, -68)])
def test_exponent(amax, e):
    assert CO.exponent(amax) == e


def test_rotation_is_a_rotation():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 576))
    y = CO.rotate(x, [0, 1, 70000], 10000.0)
    np.testing.assert_array_equal(y[:, :512], x[:, :512])
    np.testing.assert_array_equal(y[0], x[0])
    np.testing.assert_allclose(y[1, 512:514], [x[1, 512] * math.cos(1) - x[1, 513] * math.sin(1),
                                               x[1, 512] * math.sin(1) + x[1, 513] * math.cos(1)], rtol=1e-14)
    a = 70000 * 10000.0 ** (-2 / 64)
    np.testing.assert_allclose(y[2, 514], x[2, 514] * math.cos(a) - x[2, 515] * math.sin(a), rtol=1e-12)
    # scores of rotated pairs depend on the distance alone
    u, v = rng.standard_normal((1, 576)), rng.standard_normal((1, 576))
    s = [(CO.rotate(u, [t + 9], 1e4)[0, 512:] * CO.rotate(v, [t], 1e4)[0, 512:]).sum() for t in (0, 5, 4000)]
    np.testing.assert_allclose(s, s[0], rtol=1e-9)


def test_append_in_steps_keeps_values_within_their_rounding():
    """Tokens written one at a time: the last scale of a block is that of its largest token, and each value is
    off by at most half a step for its own rounding and, below the later scale's normal range, half a subnormal one."""
    rng = np.random.default_rng(2)
    n, P = 37, 16
    vals = (rng.standard_normal((n, 576)) * np.exp2(rng.integers(-6, 7, (n, 1)))).astype(np.float32)
    bits = C.W.f32_to_bf16_bits(vals)
    table = np.random.default_rng(0).permutation(4)[None, :3].astype(np.int32)
    data, scales = np.full((4, P, 576), C.NAN8, np.uint8), np.full((4, 1, 2), C.NAN16, np.uint16)
    for t in range(n):
        b = C.W.Batch(P, np.array([t], np.int32), np.array([1], np.int32), table, 4)
        data, scales, _ = CO.append8(b, bits[t:t + 1], 0.0, data.reshape(4, P, 576), scales.reshape(4, 1, 2))
    b = C.W.Batch(P, np.array([n], np.int32), np.array([1], np.int32), table, 4)
    got, x = CO.keys8(b, 0, n, data, scales), CO.bf16_value(bits)
    for b0 in range(0, n, 16):
        for d0, d1 in CO.PARTS:
            want = x[b0:b0 + 16, d0:d1]
            s = 2.0 ** CO.exponent(np.abs(want).max())
            # a value may be rounded once for each growth; only the last one in the subnormal range loses more than half a step
            assert (np.abs(got[b0:b0 + 16, d0:d1] - want) <= np.abs(want) * 2.0 ** -4 + 2 * s * 2.0 ** -10).all()
    # all at once
    b = C.W.Batch(P, np.array([0], np.int32), np.array([n], np.int32), table, 4)
    d1, s1, touched = CO.append8(b, bits, 0.0, np.full((4, P, 576), C.NAN8, np.uint8), np.full((4, 1, 2), C.NAN16, np.uint16))
    np.testing.assert_array_equal(s1[table[0]], scales.reshape(-1, 2)[table[0]])
    assert len(touched) == 2 * n
    spare = [p for p in range(4) if p not in table[0]][0]
    assert (d1.reshape(4, P, 576)[spare] == C.NAN8).all() and (d1.reshape(4, P, 576)[table[0, 2], 5:] == C.NAN8).all()


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 3), (5, 0), (5, 2), (100, 7), (3, 100)])
def test_visible(window, sinks):
    for pos in (0, 1, 4, 5, 6, 40):
        mask = [(j <= pos) and (not window or pos - j < window or j < sinks) for j in range(pos + 3)]
        assert CO.visible(pos, window, sinks) == [j for j in range(pos + 3) if mask[j]]


def test_attention_matches_the_step_oracle():
    import oracle
    wl = C.W.custom([20, 0, 7], [1, 9, 3], page_size=16, seed=5)
    li = wl.layer(0)
    pool, out, lse = oracle.step(wl.batch, li, C.W.SOFTMAX_SCALE)
    got, gl = CO.attend(wl.batch, li.q, lambda r, n: CO.keys16(wl.batch, r, n, pool), C.W.SOFTMAX_SCALE)
    np.testing.assert_allclose(got, out, rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(gl, lse, rtol=1e-12)
    wide, wl_ = CO.attend(wl.batch, li.q, lambda r, n: CO.keys16(wl.batch, r, n, pool), C.W.SOFTMAX_SCALE, window=30)
    np.testing.assert_array_equal(wide, got)
