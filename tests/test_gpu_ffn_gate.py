"""silu of the block's gate over its whole range (needs an MI355X): inside the range of exp, where
the quotient is tiny, and beyond both ends."""
import numpy as np
import pytest
import torch

from ffn_cases import Matrix, ffn
from harness import log
from test_gpu_ffn_h import DOWN, U

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HIDDEN = INNER = 96
LAST = -88.71875  # exp(-g) is a finite fp32 down to here
FACTORS = (1.0, -1.0, 0.5, -0.5, 1.5, -1.5)


def inputs(T):
    """(x, v): x[t][0] + x[t][1] is v[t], a multiple of 1 / 64, and x[t][2] is 1."""
    v = np.round(np.linspace(0, 104, T) * 64) / 64
    v[0] = 88.5
    special = [87.25, 87.328125, 87.34375, 87.375, 87.5, 58.234375, 58.25, 59.125, 88.703125, 88.71875, 0.015625, 200.0, 300.0, 1000.0]
    if T > len(special):
        v[1:1 + len(special)] = special
    x = np.zeros((T, HIDDEN))
    high = torch.from_numpy(v).to(BF16)
    x[:, 0], x[:, 1], x[:, 2] = high.double().numpy(), v - high.double().numpy(), 1.0
    x = torch.from_numpy(x)
    assert torch.equal(x.to(BF16).double(), x)
    return x.to(BF16), v


def weights(four):
    """gate i is factor[i] v, up i is scale[i]; output 2 j is 2^DOWN h[2 j], output 2 j + 1 infinite times h[2 j]."""
    i = np.arange(INNER)
    factor, exponent = np.array(FACTORS)[i // 2 % len(FACTORS)], np.where(i // 2 % 7 < 3, 0, 64)
    gate, up, down = mats = [Matrix(1, INNER, HIDDEN, four) for _ in range(3)]
    if not four:
        for m in mats:
            m.w[:] = 0
        gate.w[:, :2] = torch.from_numpy(factor).to(BF16)[:, None]
        up.w[:, 2] = torch.from_numpy(2.0 ** exponent).to(BF16)
        down.w[i, i // 2 * 2] = torch.from_numpy(np.where(i % 2 == 1, np.inf, 2.0 ** DOWN)).to(BF16)
        return mats, factor, exponent
    for m in mats:
        m.codes[:], m.scales[:] = 0, 127
    code = (np.abs(factor) * 2).astype(np.int64) + 8 * (factor < 0)
    gate.codes[:, 0] = torch.from_numpy(code * 17).to(torch.uint8)
    up.codes[:, 1], up.scales[:, 0] = 0x02, torch.from_numpy(127 + exponent).to(torch.uint8)
    down.codes[i, i // 2] = torch.from_numpy(np.where(i % 2 == 1, 7, 2)).to(torch.uint8)  # (k = 2 (i / 2): the low half)
    down.scales[:] = torch.from_numpy(np.where(i % 2 == 1, 254, 127 + DOWN)).to(torch.uint8)[:, None]
    return mats, factor, exponent


@pytest.mark.parametrize("four", [False, True], ids=["bf16w", "mx4"])
@pytest.mark.parametrize("T", [1, 17, 64, 300, 1100])
def test_silu(T, four):
    """Within 2^-21 of itself down to -88.72, where it is 2^-121.5, not 0: an infinite weight makes it an infinity.  Further down
    exp is infinite and silu may be 0.  h adds a rounding of fp32 (2^-24, or half a step of 2^-149) and, below 2^-110, half a U."""
    log(f"[gpu] silu, {T} rows, {four}")
    x, v = inputs(T)
    mats, factor, exponent = weights(four)
    got = ffn(x, mats, F32)
    g = v[:, None] * factor
    with np.errstate(over="ignore"):
        h = g / (1.0 + np.exp(-g)) * 2.0 ** exponent
    inside = g >= LAST
    bound = np.where(inside, (2.0 ** -21 + 2.0 ** -24) * np.abs(h) + 2.0 ** -150 + np.where(np.abs(h) < 2.0 ** -110, U / 2, 0), np.abs(h))
    bound[g == 0] = 0
    off, even = np.abs(got * 2.0 ** -DOWN - h), np.arange(INNER) % 2 == 0
    bad = (off > bound) & even
    assert not bad.any(), f"{int(bad.sum())} values, gates {sorted(set(g[bad].tolist()))[:6]}"
    want = np.where(g == 0, np.nan, np.copysign(np.inf, h))
    where = inside & ~even
    assert np.array_equal(got[where], want[where], equal_nan=True), f"infinities: gates {sorted(set(g[where & (got != want)].tolist()))[:6]}"
