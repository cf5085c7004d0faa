"""The block's gated values h in front of fp32 output (needs an MI355X): held in three bf16
parts of one sign, none of them zero unless h is.

The sum of the parts is h from 2^-110 on, below it h to a multiple of U = 2^-133, the least
part; a nonzero h counts as 3 U at least."""
import numpy as np
import pytest
import torch

from ffn_cases import Matrix, ffn
from harness import log
from test_gpu_ffn import EVERY_KERNEL

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -133
DOWN = 24  # the down projection's weights are 2^24, so that outputs of the smallest h are normal numbers
# (4-bit weights, rows, hidden, inner): small ones, and those that between them take every kernel in front of fp32 output
SHAPES = [(four, T, 192, 96) for four in (False, True) for T in (1, 17, 40, 300)]
SHAPES += [(what == 2, T, k, n) for what, T, k, n, f32 in EVERY_KERNEL if what != 0 and f32]


def inputs(T, hidden):
    """(x, m): x[t][1] + x[t][2] + x[t][3] is m[t], a number of up to 24 bits in (-2, 2); x[t][0] is 1."""
    rng = np.random.default_rng([71, T])
    part = rng.integers(0, 256, (T, 3))
    part[:, 0] = rng.integers(128, 256, T)
    if T >= 16:  # one part alone, two, bits at both ends, a power of two, its neighbours, nothing
        part[:7] = [[200, 0, 0], [200, 77, 0], [128, 0, 1], [128, 0, 0], [255, 255, 255], [128, 1, 0], [0, 0, 0]]
    sign = np.where(rng.integers(0, 2, T) == 1, -1.0, 1.0)
    x = np.zeros((T, hidden))
    x[:, 0] = 1.0
    x[:, 1:4] = part * sign[:, None] * 2.0 ** np.array([-7, -15, -23])
    return torch.from_numpy(x).to(BF16), x[:, 1:4].sum(axis=1)


def picks(hidden, inner):
    """Of which h an output column is a multiple: columns 2 j and 2 j + 1 of the same one."""
    return np.arange(hidden) // 2 * 37 % inner


def weights(exponents, gate_exponent, hidden, four):
    """Row i of the gate projection is 2^gate_exponent x[0], of the up projection 2^exponents[i] (x[1] + x[2] + x[3]); even
    outputs are 2^DOWN times their h, odd ones infinite times it."""
    inner = len(exponents)
    mats = [Matrix(1, n, k, four) for n, k in ((inner, hidden), (inner, hidden), (hidden, inner))]
    gate, up, down = mats
    n, i = np.arange(hidden), picks(hidden, inner)
    odd = n % 2 == 1
    if not four:
        for m in mats:
            m.w[:] = 0
        gate.w[:, 0] = 2.0 ** gate_exponent
        up.w[:, 1:4] = torch.from_numpy(2.0 ** exponents).to(BF16)[:, None]
        down.w[n, i] = torch.from_numpy(np.where(odd, np.inf, 2.0 ** DOWN)).to(BF16)
        return mats
    for m in mats:
        m.codes[:], m.scales[:] = 0, 127
    gate.codes[:, 0], gate.scales[:, 0] = 0x02, 127 + gate_exponent
    up.codes[:, 0], up.codes[:, 1], up.scales[:, 0] = 0x20, 0x22, torch.from_numpy(127 + exponents).to(torch.uint8)
    down.codes[n, i // 2] = torch.from_numpy(np.where(odd, 7, 2) << (4 * (i % 2))).to(torch.uint8)  # 6 and 1
    down.scales[n] = torch.from_numpy(np.where(odd, 254, 127 + DOWN)).to(torch.uint8)[:, None]
    return mats


def check(got, h, bound):
    """Even columns of `got` are 2^DOWN h within the bound, odd ones infinite with h's sign."""
    off = np.abs(got[:, 0::2] * 2.0 ** -DOWN - h[:, 0::2])
    bad = off > bound[:, 0::2]
    assert not bad.any(), f"{int(bad.sum())} of {bad.size}, |h| up to 2^{np.log2(np.abs(h[:, 0::2])[bad].max()):.1f}, off by up to {(off[bad] / U).max():.3g} U"
    odd = h[:, 1::2]
    assert np.array_equal(got[:, 1::2], np.where(odd == 0, np.nan, np.copysign(np.inf, odd)), equal_nan=True)


@pytest.mark.parametrize("four,T,hidden,inner", SHAPES)
def test_h_keeps_24_bits(four, T, hidden, inner):
    """Gates of 256 are their own silu, so h = 256 u, here with up to 24 bits and 2^-118 <= |h| < 2^90.  A product of h with a
    power of two is exact: each partial sum of the parts is a multiple of h's last bit and no larger than h."""
    log(f"[gpu] h of 24 bits, {T} x {hidden} x {inner}, {four}")
    x, m = inputs(T, hidden)
    exponents = np.round(np.linspace(-126, 80, inner)).astype(np.int64)
    got = ffn(x, weights(exponents, 8, hidden, four), F32)
    h = m[:, None] * 2.0 ** (exponents[picks(hidden, inner)] + 8.0)
    check(got, h, np.where(np.abs(h) >= 2.0 ** -110, 0.0, U / 2) * (h != 0))


@pytest.mark.parametrize("four,T,hidden,inner", SHAPES)
def test_smallest_h(four, T, hidden, inner):
    """Gates of 2^-60, whose silu is 2^-61 (1 + exp(-g) is 2), and |h| from 2^-72 down to 2^-140.  silu is off by 2^-21 of
    itself at most, its product with u by half of fp32's least step, 2^-150; then h to half a U, and below 3 U to 3 U."""
    log(f"[gpu] smallest h, {T} x {hidden} x {inner}, {four}")
    x, m = inputs(T, hidden)
    exponents = np.round(np.linspace(-79, -12, inner)).astype(np.int64)
    got = ffn(x, weights(exponents, -60, hidden, four), F32)
    h = m[:, None] * 2.0 ** (exponents[picks(hidden, inner)] - 61.0)
    check(got, h, (np.abs(h) * 2.0 ** -21 + 2.0 ** -150 + np.where(np.abs(h) < 3 * U, 3 * U, U / 2)) * (h != 0))
