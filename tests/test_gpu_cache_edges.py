"""The compact latent cache on the GPU at the edges of its contract: pools that end
inside a 16-byte piece of the scales, and what else a caller may rely on there."""
import numpy as np
import pytest

import cache_cases as C
import paper_2607_02043_amd as mla
from harness import log, to_dev
from oracle import cache_oracle as CO
from paper_2607_02043_amd import workloads as W
from test_gpu_cache import BASE, SCALE, Attend, down8, flags, up8  # noqa: F401  (flags: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [None, (20, 2)], ids=str)
@pytest.mark.parametrize("prefix,rows", [([3], [1]), ([0], [14]), ([17, 0], [1, 1]), ([30, 0, 5], [1, 9, 1])], ids=str)
def test_scales_that_end_inside_a_piece(prefix, rows, window):
    """Pools of 1, 2, 3, .. blocks, their scales at the very end of an allocation."""
    import torch
    b = C.batch(prefix, rows, 16, seed=41)
    need = int(b.block_table.max()) + 1
    for pages in (need, need + 1, need + 2, need + 3):
        log(f"[gpu] {prefix} {rows}, {pages} blocks, window {window}")
        b.num_pages = pages
        data, scales = C.cache8(b, 2, upto=lambda r: int(b.prefix_lens[r] + b.q_lens[r]))
        a = Attend(b, C.queries(b, 1), data, scales, window=window)
        whole = torch.full((8 + 2 * pages,), float("nan"), dtype=torch.bfloat16, device="cuda")
        own = whole[8:].view(pages, 1, 2)
        own.view(torch.int16).copy_(to_dev(scales))
        a.cache = mla.LatentCache8(data=up8(data), scales=own)
        a.run().check(f"{pages} blocks")
    assert mla.device_flags() == 0


def top_codes(data):
    """Codes of at most 240, the largest whose value times 2^120 a bf16 holds; NaN stays."""
    mag = data & 0x7F
    return np.where((mag > 0x77) & (mag < 0x7F), (data & 0x80) | 0x77, data).astype(np.uint8)


@pytest.mark.parametrize("spread", [0.0, 1.0], ids=["equal scores", "own scores"])
@pytest.mark.parametrize("prefix,rows,keys,unit", [([700], [1], 0, 1), ([2500, 90], [1, 1], 0, 3), ([300], [20], 64, 0),
                                                   ([1500, 0], [9, 33], 128, 0), ([20000], [2], 64, 0)], ids=str)
def test_split_rows_of_the_largest_values(prefix, rows, keys, unit, spread):
    """Every compressed scale 2^120, where a sum over keys that are equally likely is far beyond fp32 and their average
    is not: rows whose keys are split over units and ranges, and those that are not."""
    b = C.batch(prefix, rows, 64, seed=42)
    data, scales = C.cache8(b, 7, upto=lambda r: int(b.prefix_lens[r] + b.q_lens[r]))
    scales = scales.copy()
    nan = scales[..., 0] == C.NAN16
    scales[..., 0] = np.where(nan, C.NAN16, CO.scale_bits(np.array([120]))[0])
    q = C.queries(b, 3, scale=spread).reshape(-1, 16, 576)
    q[:, :, :512] = 0  # scores come from the rope dims alone
    for k, u in ((keys, unit), (0, 1 << 20)):
        mla.debug_set(mla.MLA_DEBUG_CHUNK_KEYS, k)
        mla.debug_set(mla.MLA_DEBUG_DEC_UNIT, u)
        log(f"[gpu] {prefix} {rows}, chunk keys {k}, unit {u}")
        Attend(b, q, top_codes(data), scales).run().check("largest values", range(0, b.num_rows, 3))
    assert mla.device_flags() == 0


@pytest.mark.parametrize("base", [0.0, BASE])
def test_append8_of_the_largest_finite_values(base):
    """bf16 values next to 2^128: codes whose values a bf16 holds, off by half a step at most."""
    b = C.batch([0, 5, 16], [16, 2, 1], 16, seed=43)
    new = C.new_latents(b, 4).copy()
    tops = np.array([0x7F7F, 0xFF7F, 0x7F78, 0x7F77, 0xFF70, 0x7F6F, 0x7F00], dtype=np.uint16)
    new[0, 3:3 + len(tops)] = tops
    new[16, 100], new[18, 500] = 0x7F7F, 0xFF7F
    new[9, 512:576:2], new[9, 513:576:2] = 0x7F7F, 0  # (one of a pair: rotated it stays below 2^128)
    data, scales = C.cache8(b, 2)
    c = mla.LatentCache8(num_pages=b.num_pages, page_size=16)
    import torch
    c.data.copy_(up8(data))
    c.scales.view(torch.int16).copy_(to_dev(scales))
    db = mla.DeviceBatch.from_batch(b)
    mla.append_latent_kv8(db, to_dev(new), c, rope_base=base)
    got, gs = down8(c)
    if not base:
        want, ws, _ = CO.append8(b, new, base, data, scales)
        np.testing.assert_array_equal(gs.reshape(-1, 2), ws)
        np.testing.assert_array_equal(got.reshape(-1, 576), want)
    for r, x in enumerate(CO.rows(b, new, base)):
        keys = CO.keys8(b, r, int(b.prefix_lens[r] + b.q_lens[r]), got, gs)[int(b.prefix_lens[r]):]
        s = np.array([[CO.scale_value(gs.reshape(-1, 2)[CO.slot(b, r, int(b.prefix_lens[r]) + i) // 16, k]) for k in (0, 1)] for i in range(len(x))])
        half = np.concatenate((np.repeat(s[:, :1], 512, 1), np.repeat(s[:, 1:], 64, 1)), 1) * 2.0 ** -10
        m = np.zeros_like(x)  # (rotated in fp32: cos and sin within 2^-22, two products and a sum)
        m[:, 512:] = np.repeat(np.abs(CO.bf16_value(new)[int(b.cu_q[r]):int(b.cu_q[r + 1]), 512:]).reshape(len(x), 32, 2).sum(2), 2, 1) * 2.0 ** -21
        assert (np.abs(keys) < 2.0 ** 128).all()  # NaN and infinities fail it
        assert (np.abs(keys - x) <= np.abs(x) * 2.0 ** -4 + half + m).all()
    # and read back: attention gives finite rows
    a = Attend(b, C.queries(b, 1).reshape(-1, 16, 576) * np.uint16(0), *down8(c))
    a.run().check("largest values")


@pytest.mark.parametrize("keys,unit", [(0, 0), (64, 1)], ids=["whole", "split"])
@pytest.mark.parametrize("window", [(16, 2), (70, 3), (1 << 20, 0)], ids=str)
def test_infinities_of_a_windowed_cache(window, keys, unit):
    """An infinite cached value whose score is -inf has a weight of 0, and 0 x inf is NaN: in that value's dim of every
    row that sees the key, wherever its tile lies, and nowhere else.  Infinite rope dims have a weight of 0 alone."""
    b = C.batch([50, 20, 33, 150], [1, 90, 1, 40], 32, seed=44)
    pool, q = filled(b, 5), C.queries(b, 1).reshape(-1, 16, 576)
    NEG, INF = 0xBF80, 0x7F80
    q[:, :, 100], q[:, 5, 100] = NEG, 0x3F80  # scores of the values below: -inf, +inf for head 5
    q[:, :, 300] = q[:, :, 7] = q[:, :, 530] = NEG
    flat = pool.reshape(-1, 576)
    for r, t, d in ((0, 45, 100), (0, 50, 300), (1, 30, 100), (1, 75, 300), (1, 75, 7), (2, 3, 100), (2, 1, 300), (3, 160, 300), (3, 0, 300), (3, 63, 100)):
        flat[CO.slot(b, r, t), d] = INF
    for r, t in ((1, 40), (0, 48), (3, 170)):
        flat[CO.slot(b, r, t), 530] = INF
    mla.debug_set(mla.MLA_DEBUG_CHUNK_KEYS, keys)
    mla.debug_set(mla.MLA_DEBUG_DEC_UNIT, unit)
    a = Attend(b, q, pool=pool, window=window).run()
    out, lse = a.results()
    qv = CO.bf16_value(q)
    for row in range(b.num_rows):
        r = int(np.searchsorted(b.cu_q, row, side="right")) - 1
        pos = int(b.prefix_lens[r]) + row - int(b.cu_q[r])
        k = CO.keys16(b, r, pos + 1, pool)
        with np.errstate(invalid="ignore"):
            ro, rl = CO.attend_row(qv[row], k, pos, SCALE, *window)
        nan = np.isnan(ro)
        np.testing.assert_array_equal(np.isnan(out[row]), nan, err_msg=str((r, pos)))
        # what is finite, against bounds without the keys of weight 0
        few = k[[j for j in CO.visible(pos, *window) if np.isfinite(k[j]).all()]]
        to, tl = C.bounds(qv[row], few, len(few) - 1, SCALE, 0, 0, b.q_lens[r] > 1, not a.bf16, np.where(nan, 0, ro), np.where(np.isnan(rl), 0, rl))
        assert (np.where(nan, 0, np.abs(out[row] - ro)) <= to).all(), (r, pos)
        assert (np.where(np.isnan(rl), 0, np.abs(lse[row] - rl)) <= tl).all(), (r, pos)


def filled(b, seed):
    """A bf16 pool with all of every request's tokens."""
    rng = np.random.default_rng([seed, 4])
    return W.f32_to_bf16_bits(rng.standard_normal((b.num_pages * b.page_size, 576), dtype=np.float32)).reshape(b.num_pages, b.page_size, 576)


@pytest.mark.parametrize("stale", ["outside the pool", "another request's"])
@pytest.mark.parametrize("kind", ["8-bit", "rotated", "bf16"])
def test_check_mode_of_a_windowed_program_that_gives_pages_back(kind, stale):
    """Entries of pages that no row sees any more hold anything: an append then attends under check mode as without."""
    import torch
    window, P = (40, 5), 16
    b = C.batch([300, 200, 90], [1, 33, 1], P, seed=45)
    q, new = C.queries(b, 1), to_dev(C.new_latents(b, 3))
    data, scales = C.cache8(b, 2)
    bt = b.block_table.copy()
    for r in range(b.num_reqs):
        for lp in range(bt.shape[1]):
            if lp * P >= window[1] and lp * P + P - 1 <= int(b.prefix_lens[r]) - window[0]:
                # (the page that the next request writes its first new token into)
                o = (r + 1) % b.num_reqs
                bt[r, lp] = (-3, b.num_pages, 1 << 30)[lp % 3] if stale == "outside the pool" else b.block_table[o, int(b.prefix_lens[o]) // P]
    results = []
    for check, table in ((0, b.block_table), (0, bt), (1, bt)):
        mla.debug_set(mla.MLA_DEBUG_CHECK, check)
        a = Attend(b, q, data, scales, window=window) if kind == "8-bit" else Attend(b, q, pool=filled(b, 5), window=window)
        a.db.bt_dev.copy_(torch.from_numpy(table))
        if kind == "8-bit":
            mla.append_latent_kv8(a.db, new, a.cache, rope_base=BASE)
        elif kind == "rotated":
            mla.append_latent_kv_rope(a.db, new, BASE, a.cache)
        else:
            mla.append_latent_kv(a.db, new, a.cache)
        results.append(a.run().results())
    for x in results[1:]:
        for u, v in zip(results[0], x):
            np.testing.assert_array_equal(u, v)
    assert mla.device_flags() == 0
    # what an append writes into is still looked at
    a.db.bt_dev[1, 210 // P] = b.num_pages
    call = {"8-bit": lambda: mla.append_latent_kv8(a.db, new, a.cache), "rotated": lambda: mla.append_latent_kv_rope(a.db, new, BASE, a.cache),
            "bf16": lambda: mla.append_latent_kv(a.db, new, a.cache)}[kind]
    with pytest.raises(mla.MlaError, match="outside"):
        call()


def fine_bounds(x_max, n, v, top, ref):
    """How far an fp32 output may be from the 64-bit one where a score is one exact product s: x = s scale log2(e) in
    fp32 (two roundings of 2^-24 |x|, one more of the difference to the reference), exp2 within 2^-22, the sums of
    cache_cases.bounds.  Probabilities as fp16 hi + lo: 2^-22 of p, and 2^-25 where lo is below fp16's normal
    range, each key once; the largest p is at least 2^6, so 2^-31 of the sum.  A bf16 value goes to fp16 within
    2^-24, one of the 8-bit cache within 2^-25 of `top`."""
    delta = 2.0 ** -24 * 3 * x_max * np.log(2) + 2.0 ** -22
    sums = 2.0 ** -24 * (n / 8 + 8)
    return v * (2 * delta + 2.0 ** -22 + n * 2.0 ** -31 + 2 * sums) + (2.0 ** -25 * top if top else 2.0 ** -24) + 2.0 ** -24 * np.abs(ref)


@pytest.mark.parametrize("keys", [0, 64], ids=["whole", "split"])
@pytest.mark.parametrize("window", [None, (12, 3), (100, 0)], ids=str)
@pytest.mark.parametrize("eight", [True, False], ids=["8-bit", "bf16"])
def test_fp32_output_of_chunk_rows(eight, window, keys):
    """Chunk rows with fp32 output hold more of a probability than an fp16 has."""
    window = window if eight or window else (1 << 20, 0)
    b = C.batch([0, 37, 150, 64], [40, 21, 30, 1], 16, seed=46)
    q = np.zeros((b.num_rows, 16, 576), np.uint16)
    q[:, :, 575] = W.f32_to_bf16_bits(np.random.default_rng(46).uniform(-32, 32, (b.num_rows, 16)).astype(np.float32))
    mla.debug_set(mla.MLA_DEBUG_CHUNK_KEYS, keys)
    if eight:
        a = Attend(b, q, *C.cache8(b, 2, upto=lambda r: int(b.prefix_lens[r] + b.q_lens[r])), window=window)
    else:
        a = Attend(b, q, pool=filled(b, 5), window=window)
    out, _ = a.run().results()
    qv = CO.bf16_value(q)
    off = base = 0.0
    for row in range(b.num_rows - 1):
        r = int(np.searchsorted(b.cu_q, row, side="right")) - 1
        i = row - int(b.cu_q[r])
        pos = int(b.prefix_lens[r]) + i
        k = a.keys(r, pos + 1)
        ro, _ = CO.attend_row(qv[row], k, pos, SCALE, *(window or (0, 0)))
        seen = k[CO.visible(pos, *(window or (0, 0)))]
        x = np.abs(qv[row, :, 575]).max() * np.abs(seen[:, 575]).max() * SCALE * np.log2(np.e)
        lim = fine_bounds(x, len(seen), np.abs(seen[:, :512]).max(), a.top_scale(r, i), ro)
        assert (np.abs(out[row] - ro) <= lim).all(), (r, pos, float((np.abs(out[row] - ro) / lim).max()))
        off, base = off + ((out[row] - ro) ** 2).sum(), base + (ro ** 2).sum()
    log(f"  relative error {np.sqrt(off / base):.2e}")
    assert mla.device_flags() == 0


@pytest.mark.parametrize("eight,window", [(True, None), (True, (1 << 20, 0)), (False, (1 << 20, 0))], ids=str)
@pytest.mark.parametrize("prefix", [1, 3, 9, 40])
def test_fp32_output_of_decode_rows(prefix, eight, window):
    """Decode rows in the 2-norm.  A weight off by e_j moves the output by w_j e_j (v_j - out); the values here are
    independent with mean 0, so over many rows and dims the error's norm is at most max |e| of the output's.
    e, in 2^-24: the score, one product and x = s scale log2(e), three roundings of |x| ln 2 (|x| < 1.6 but for a few:
    4 x 3.5 x SCALE log2 e); exp2 within an ulp, 2; the probability's parts 2^-22, 4; the sum, its inverse and the output, 3."""
    b = C.batch([prefix] * 40, [1] * 40, 16, seed=47)
    q = np.zeros((b.num_rows, 16, 576), np.uint16)
    q[:, :, 575] = W.f32_to_bf16_bits(np.random.default_rng(47).uniform(-4, 4, (b.num_rows, 16)).astype(np.float32))
    if eight:
        a = Attend(b, q, *C.cache8(b, 2, upto=lambda r: prefix + 1), window=window)
    else:
        a = Attend(b, q, pool=filled(b, 5), window=window)
    out, _ = a.run().results()
    want = np.stack([CO.attend_row(CO.bf16_value(q[r]), a.keys(r, prefix + 1), prefix, SCALE)[0] for r in range(40)])
    rel = np.sqrt(((out - want) ** 2).sum() / (want ** 2).sum())
    log(f"  relative error {rel:.2e}")
    assert rel <= 2.0 ** -24 * (3 * 1.6 * np.log(2) + 2 + 4 + 3)
