"""Pins of the feed-forward oracle (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import ffn_oracle as O


def test_mx4_values_of_every_code_and_scale():
    codes = np.arange(256, dtype=np.uint8).reshape(16, 16)
    flat = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    for b in (0, 1, 100, 127, 128, 252):
        v = O.mx4_values(codes, np.full((16, 1), b, dtype=np.uint8))
        for byte in range(256):
            for j, c in enumerate((byte % 16, byte // 16)):
                want = (-1 if c >= 8 else 1) * flat[c % 8] * 2.0 ** (b - 127)
                assert v[byte // 16, 2 * (byte % 16) + j] == want
    assert np.isnan(O.mx4_values(codes, np.full((16, 1), 255, dtype=np.uint8))).all()
    top = O.mx4_values(codes, np.full((16, 1), 253, dtype=np.uint8))
    # magnitudes 4 and 6 of either sign, 32 of the 512 codes each
    assert np.isinf(top).sum() == 4 * 32 and np.abs(top[np.isfinite(top)]).max() == 3 * 2.0 ** 126


def test_values_below_2_to_128_are_exact_in_bf16():
    codes = np.tile(np.arange(16, dtype=np.uint8), (254, 1))
    v = O.mx4_values(codes, np.arange(254, dtype=np.uint8)[:, None])
    v = np.where(np.isinf(v), 0.0, v)
    assert np.array_equal(torch.from_numpy(v).to(torch.bfloat16).double().numpy(), v)


def test_quantize_is_the_nearest_value():
    w = np.random.default_rng(0).standard_normal((5, 96))
    codes, scales = O.mx4_quantize(w)
    v = O.mx4_values(codes, scales)
    s = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=1)
    assert np.all(np.abs(v - w) <= s) and np.all(np.abs(w) <= 6 * s) and np.all(np.abs(w).reshape(5, 3, 32).max(2) > 3 * s[:, ::32])


def test_block_against_plain_loops():
    rng = np.random.default_rng(1)
    x, gate, up, down = (rng.standard_normal(s) for s in ((3, 5), (4, 5), (4, 5), (5, 4)))
    out, bound = O.ffn(x, gate, up, down, 1)
    for t in range(3):
        h = []
        for i in range(4):
            g = sum(x[t, k] * gate[i, k] for k in range(5))
            h.append(g / (1 + math.exp(-g)) * sum(x[t, k] * up[i, k] for k in range(5)))
        for n in range(5):
            assert out[t, n] == pytest.approx(sum(h[i] * down[n, i] for i in range(4)), rel=1e-12)
    assert np.all(bound > 0) and np.all(O.rounded_bound(out, bound, True) > bound)


@pytest.mark.parametrize("planes", [1, 3])
def test_bound_covers_fp32_arithmetic_and_sees_a_mistake(planes):
    rng = np.random.default_rng(2)
    x, gate, up, down = (torch.from_numpy(rng.standard_normal(s) / math.sqrt(s[1])).to(torch.bfloat16)
                         for s in ((7, 256), (96, 256), (96, 256), (256, 96)))
    out, bound = O.ffn(*(t.double().numpy() for t in (x, gate, up, down)), planes)
    g, u = x.float() @ gate.float().T, x.float() @ up.float().T
    h = g / (1 + torch.exp(-g)) * u
    h = h.to(torch.bfloat16).float() if planes == 1 else h
    y = (h @ down.float().T).double().numpy()
    assert np.all(np.abs(y - out) <= bound)
    # one weight of the up projection missing, as a tail that is cut off would
    up0 = up.clone()
    up0[:, -8:] = 0
    wrong, _ = O.ffn(*(t.double().numpy() for t in (x, gate, up0, down)), planes)
    assert np.mean(np.abs(wrong - out) > O.rounded_bound(out, bound, planes == 1)) > 0.2
