"""Plain numpy fp64 oracle of the compact latent cache: the rotation of appended
latents, the 8-bit cache (e4m3 codes, two power-of-two scales for every block of
16 tokens) and attention through a window with sinks.

TEST INFRASTRUCTURE ONLY: it shares no code, table or constant with the HIP
library; the shapes and rules are restated here on purpose.
"""
import math

import numpy as np

HEADS, DQK, DV, BLOCK = 16, 576, 512, 16
PARTS = ((0, 512), (512, 576))
E_MIN, E_MAX = -100, 120


def bf16_value(bits):
    return (np.asarray(bits, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def e4m3_table():
    """Value of each of the 256 codes."""
    t = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        v = math.nan if e == 15 and m == 7 else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        t[c] = -v if s else v
    return t


TABLE = e4m3_table()


def e4m3_code(v):
    """Nearest code of each value, |v| <= 448 or NaN; of two as near, the one with an even mantissa."""
    v = np.asarray(v, dtype=np.float64)
    pos = TABLE[:127]  # 0 .. 448 ascending, code = index
    a = np.where(np.isnan(v), 0.0, np.abs(v))
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    return np.where(np.isnan(v), np.uint8(0x7F), np.where(np.signbit(v), c | 0x80, c)).astype(np.uint8)


def rotate(x, pos, base):
    """x [n][576]: pairs (2i, 2i + 1) of the last 64 dims by pos base^(-2i / 64)."""
    y = np.array(x, dtype=np.float64)
    for n in range(len(y)):
        for i in range(32):
            a = float(pos[n]) * base ** (-2.0 * i / 64)
            u, w = x[n][512 + 2 * i], x[n][513 + 2 * i]
            y[n][512 + 2 * i] = u * math.cos(a) - w * math.sin(a)
            y[n][513 + 2 * i] = u * math.sin(a) + w * math.cos(a)
    return y


def exponent(amax):
    """Smallest E in range with amax 2^-E <= 448."""
    for e in range(E_MIN, E_MAX + 1):
        if amax * 2.0 ** -e <= 448.0:
            return e
    raise ValueError(amax)


def largest(e):
    """Largest e4m3 value that a bf16 holds times 2^e (448, or below 2^(128 - e))."""
    return max(v for v in TABLE[:127] if v * 2.0 ** e < 2.0 ** 128)


def scale_bits(e):
    return np.uint16((e + 127) << 7)


def scale_value(bits):
    return bf16_value(bits)


def slot(batch, r, t):
    return int(batch.block_table[r][t // batch.page_size]) * batch.page_size + t % batch.page_size


def rows(batch, new_bits, base):
    """Per request: the values that its new tokens are cached with."""
    x = bf16_value(new_bits).reshape(-1, DQK)
    out, row = [], 0
    for p, c in zip(batch.prefix_lens, batch.q_lens):
        y = x[row:row + int(c)]
        out.append(rotate(y, np.arange(int(p), int(p) + int(c)), base) if base else y)
        row += int(c)
    return out


def append8(batch, new_bits, base, data, scales):
    """data uint8 [pages][P][576], scales uint16 [pages][P / 16][2]: copies after the append, and
    the set of (slot, part) whose values were rounded (again)."""
    data, scales = data.copy().reshape(-1, DQK), scales.copy().reshape(-1, 2)
    touched = set()
    for r, x in enumerate(rows(batch, new_bits, base)):
        p, c = int(batch.prefix_lens[r]), int(batch.q_lens[r])
        for b in range(p // BLOCK, (p + c - 1) // BLOCK + 1):
            t0, t1 = max(p, b * BLOCK), min(p + c, (b + 1) * BLOCK)
            blk = slot(batch, r, b * BLOCK) // BLOCK
            for k, (d0, d1) in enumerate(PARTS):
                new = x[t0 - p:t1 - p, d0:d1]
                fin = np.abs(new[np.isfinite(new)])
                e = exponent(float(fin.max()) if fin.size else 0.0)
                if t0 > b * BLOCK:
                    was = int(round(math.log2(scale_value(scales[blk, k]))))
                    e = max(e, was)
                    for t in range(b * BLOCK, t0):
                        s = slot(batch, r, t)
                        if e != was:
                            data[s, d0:d1] = e4m3_code(TABLE[data[s, d0:d1]] * 2.0 ** (was - e))
                            touched.add((s, k))
                scales[blk, k] = scale_bits(e)
                for t in range(t0, t1):
                    v = new[t - t0]
                    s = slot(batch, r, t)
                    data[s, d0:d1] = e4m3_code(np.clip(np.where(np.isfinite(v), v, math.nan) * 2.0 ** -e, -largest(e), largest(e)))
                    touched.add((s, k))
    return data, scales, touched


def keys8(batch, r, n, data, scales):
    """Values of keys 0 .. n - 1 of request r."""
    data, scales = data.reshape(-1, DQK), scales.reshape(-1, 2)
    s = np.array([slot(batch, r, t) for t in range(n)], dtype=np.int64)
    v = TABLE[data[s]]
    for k, (d0, d1) in enumerate(PARTS):
        v[:, d0:d1] *= scale_value(scales[s // BLOCK, k])[:, None]
    return v


def keys16(batch, r, n, pool):
    s = np.array([slot(batch, r, t) for t in range(n)], dtype=np.int64)
    return bf16_value(pool.reshape(-1, DQK)[s])


def visible(pos, window, sinks):
    """Keys that a row at `pos` sees (window 0: all earlier ones and its own)."""
    return [j for j in range(pos + 1) if not window or j > pos - window or j < sinks]


def attend_row(q, keys, pos, scale, window=0, sinks=0):
    """q [16][576]; keys of the request; out [16][512] and lse [16]."""
    at = visible(pos, window, sinks)
    k = keys[at]
    s = scale * (q @ k.T)
    m = s.max(axis=1)
    w = np.exp(s - m[:, None])
    return (w @ k[:, :DV]) / w.sum(axis=1)[:, None], m + np.log(w.sum(axis=1))


def attend(batch, q_bits, keys_of, scale, window=0, sinks=0, row_ids=None):
    """out [n][16][512] and lse [n][16] of the rows `row_ids` (all by default); keys_of(r, n)."""
    q = bf16_value(q_bits).reshape(-1, HEADS, DQK)
    cu = batch.cu_q
    want = list(range(batch.num_rows)) if row_ids is None else list(row_ids)
    out, lse, cache = np.empty((len(want), HEADS, DV)), np.empty((len(want), HEADS)), {}
    for n, row in enumerate(want):
        r = int(np.searchsorted(cu, row, side="right")) - 1
        if r not in cache:
            cache = {r: keys_of(r, int(batch.prefix_lens[r] + batch.q_lens[r]))}
        out[n], lse[n] = attend_row(q[row], cache[r], int(batch.prefix_lens[r]) + row - int(cu[r]), scale, window, sinks)
    return out, lse
