"""Pins of the compact cache's oracle at the ends of its ranges (CPU)."""
import numpy as np

import cache_cases as C
from oracle import cache_oracle as CO


def test_every_finite_bf16_is_held():
    """Each finite bf16 value alone in a block: its code times its scale is below 2^128 and within half a step
    (2^-4 of it, or half a subnormal step of the smallest scale)."""
    mags = np.arange(0, 0x7F80, dtype=np.uint16)
    x = CO.bf16_value(mags)
    e = np.array([CO.exponent(float(v)) for v in x])
    code = CO.e4m3_code(np.minimum(x * 2.0 ** -e, [CO.largest(int(k)) for k in e]))
    got = CO.TABLE[code] * 2.0 ** e
    assert (got < 2.0 ** 128).all()
    assert (np.abs(got - x) <= np.maximum(x * 2.0 ** -4, 2.0 ** (CO.E_MIN - 10))).all()
    # and each is a bf16: 8 significant bits
    m, _ = np.frexp(got)
    assert (m * 256 == np.round(m * 256)).all()


def test_append_of_the_largest_values():
    b = C.batch([0], [3], 16, seed=1)
    bits = np.zeros((3, 576), np.uint16)
    bits[0, 0], bits[1, 5], bits[2, 570], bits[2, 571] = 0x7F7F, 0xFF78, 0x7F7F, 0x7F80
    data, scales, _ = CO.append8(b, bits, 0.0, *C.cache8(b, 1))
    k = CO.keys8(b, 0, 3, data, scales)
    assert k[0, 0] == 240 * 2.0 ** 120 and k[1, 5] == -240 * 2.0 ** 120 and k[2, 570] == 240 * 2.0 ** 120 and np.isnan(k[2, 571])
