"""The feed-forward block and products with 4-bit weights in 64 bits (numpy), and
how far a result with fp32 sums may be from them."""
import numpy as np

GROUP = 32


def mx4_values(codes, scales):
    """Weights [N][K] that codes [N][K / 2] and scale bytes [N][K / 32] stand for, as a product with
    them counts them: infinite from 2^128 on."""
    codes = np.asarray(codes)
    c = np.empty((codes.shape[0], codes.shape[1] * 2), dtype=np.int64)
    c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
    e, m = (c >> 1) & 3, c & 1
    v = np.where(e == 0, 0.5 * m, np.ldexp(1.0 + 0.5 * m, e - 1))
    v = np.where(c & 8, -v, v)
    b = np.repeat(np.asarray(scales).astype(np.int64), GROUP, axis=1)
    v = np.ldexp(v, b - 127)
    v = np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v)
    return np.where(b == 255, np.nan, v)


def mx4_quantize(w):
    """(codes, scales) of weights [N][K]: each group under the smallest scale that holds it, values to the
    nearest magnitude."""
    g = np.asarray(w, dtype=np.float64).reshape(w.shape[0], -1, GROUP)
    amax = np.maximum(np.abs(g).max(axis=2), 2.0 ** -100)
    e = np.ceil(np.log2(amax / 6.0)).astype(np.int64)
    near = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    c = np.abs(np.abs(np.ldexp(g, -e[:, :, None]))[..., None] - near).argmin(axis=-1) + 8 * (g < 0)
    c = c.reshape(w.shape[0], -1).astype(np.uint8)
    return c[:, 0::2] | c[:, 1::2] << 4, (e + 127).astype(np.uint8)


def _sums(k, planes=1):
    """Of sum_k |a b|, what fp32 sums of k exact products may be off: at most 32 additions inside one
    matrix instruction, one a instruction, and 32 that join parts, each off by a step (2^-23)."""
    return (64.0 + planes * k / 32.0) * 2.0 ** -23


def linear(x, w):
    """(x w^T, bound on an fp32 result's distance)."""
    with np.errstate(invalid="ignore", over="ignore"):
        return x @ w.T, _sums(x.shape[1]) * (np.abs(x) @ np.abs(w).T)


def ffn(x, gate, up, down, planes):
    """(out, bound): h rounded to `planes` bf16 (relative 2^-8 or, for 3, 2^-24).  |silu'| < 1.1; exp, sum,
    quotient and product of the gate are off by at most 2^-21 of h together."""
    with np.errstate(invalid="ignore", over="ignore"):
        g, dg = linear(x, gate)
        u, du = linear(x, up)
        silu = g / (1.0 + np.exp(-g))
        h = silu * u
        dh = 1.1 * dg * (np.abs(u) + du) + np.abs(silu) * du + 2.0 ** -21 * np.abs(h)
        dh = dh + (2.0 ** -8 if planes == 1 else 2.0 ** -24) * (np.abs(h) + dh)
        out, _ = linear(h, down)
        return out, dh @ np.abs(down).T + _sums(h.shape[1], planes) * ((np.abs(h) + dh) @ np.abs(down).T)


def rounded_bound(out, bound, bf16):
    """The bound with the output's own rounding: half a step, 2^-8 or 2^-24 of the value."""
    return bound + (2.0 ** -8 if bf16 else 2.0 ** -24) * (np.abs(out) + bound)


def _sums_norm(k, planes=1):
    """As _sums, of all outputs together in the 2-norm, where products have random signs: each of the roundings is off by a step
    (2^-23) at most of a partial sum, which is no larger than the result in the mean, and they are independent."""
    return np.sqrt(64.0 + planes * k / 32.0) * 2.0 ** -23


def linear_norm(k):
    """Bound on |got - out| / |out| in the 2-norm for an fp32 result of random values."""
    return _sums_norm(k)


def ffn_norm(hidden, inner):
    """The same for a block whose h meets w_down with 24 bits: errors of g (|silu'| < 1.1) and u, the gate's 2^-21, h's
    2^-24, then those of the down projection."""
    return 2.1 * _sums_norm(hidden) + 2.0 ** -21 + 2.0 ** -24 + _sums_norm(inner, 3)
