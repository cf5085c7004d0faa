"""Seeded inputs and tolerances of the compact-cache tests."""
import numpy as np

from oracle import cache_oracle as CO
from paper_2607_02043_amd import workloads as W

NAN8, NAN16 = 0x7F, 0x7FC0


def batch(prefix, rows, page, seed=0, **kw):
    return W.make_batch(prefix, rows, page, seed, **kw)


def new_latents(b, seed, spread=1.0):
    """bf16 bits [T][576], rope dims three times as wide as the others."""
    rng = np.random.default_rng([seed, 1])
    x = rng.standard_normal((b.num_rows, 576), dtype=np.float32) * np.float32(spread)
    x[:, 512:] *= 3
    return W.f32_to_bf16_bits(x)


def queries(b, seed, scale=1.0):
    rng = np.random.default_rng([seed, 2])
    return W.f32_to_bf16_bits(rng.standard_normal((b.num_rows, 16, 576), dtype=np.float32) * np.float32(scale))


def cache8(b, seed, upto=None):
    """An 8-bit pool: keys 0 .. upto(r) - 1 of each request (its prefix by default) hold
    values of spread 2^-2 .. 2^2 by block, every other slot NaN codes, every other block NaN scales."""
    rng = np.random.default_rng([seed, 3])
    slots = b.num_pages * b.page_size
    data = np.full((slots, 576), NAN8, dtype=np.uint8)
    scales = np.full((slots // 16, 2), NAN16, dtype=np.uint16)
    for r in range(b.num_reqs):
        n = int(b.prefix_lens[r]) if upto is None else upto(r)
        if n == 0:
            continue
        t = np.arange(n)
        s = b.block_table[r, t // b.page_size].astype(np.int64) * b.page_size + t % b.page_size
        blocks = s[::16] // 16
        e = rng.integers(-9, -4, (len(blocks), 2))
        scales[blocks] = CO.scale_bits(e)
        data[s] = CO.e4m3_code(np.clip(rng.standard_normal((n, 576)) * 110, -448, 448))
    return data.reshape(b.num_pages, b.page_size, 576), scales.reshape(b.num_pages, b.page_size // 16, 2)


def bounds(q, keys, pos, scale, window, sinks, fp16_p, fp32_out, ref_out, ref_lse, top=0.0):
    """How far a row's out [16][512] and lse [16] may be from the 64-bit ones.

    Scores: fp32 sums of 576 exact products, 64 roundings of at most the sum of
    magnitudes in a row (the products of a matrix instruction, the chain of 18 of
    them, the scale): delta = 64 2^-24 max_j scale sum_d |q_d k_jd|.  A change of
    every score by at most delta moves a softmax average by at most
    2 delta max|v| and the log of the sum by delta.
    Probabilities: fp16 (chunk rows): half a step, 2^-11 of p, and 2^-25 where p is
    below fp16's normal range, each key once; a bf16 pair (decode rows) 2^-16.
    Values of chunk rows over the 8-bit cache: fp16 relative to a reference scale.  A code
    has 4 significant bits, so it is exact there down to fp16's normal range and a
    multiple of 2^-24 below it: off by half of that at most, 2^-25 of the reference.
    The reference is one for the 8 rows that are computed together and at most the
    largest scale that one of them sees, `top`; a softmax average of such errors is
    no larger.  (Far-apart scales alone make this term count: beside equal scales it
    is below 2^-25 / 2^-11 of the fp16 term of the probabilities.)
    Sums of n terms in fp32 on top: n 2^-24 of the sum of magnitudes, by halves
    of the tree at least, 2^-24 (n / 8 + 8).  The output rounds once (2^-24 or 2^-8)."""
    at = CO.visible(pos, window, sinks)
    k = keys[at]
    n, v = len(at), float(np.abs(k[:, :512]).max())
    delta = 64 * 2.0 ** -24 * scale * float((np.abs(q) @ np.abs(k).T).max())
    sums = 2.0 ** -24 * (n / 8 + 8)
    p = 2.0 ** -11 + n * 2.0 ** -25 if fp16_p else 2.0 ** -16
    out = v * (2 * delta + p + 2 * sums) + 2.0 ** -25 * top + np.abs(ref_out) * (2.0 ** -24 if fp32_out else 2.0 ** -8)
    return out, delta + sums + 2.0 ** -22 * (1 + np.abs(ref_lse))
