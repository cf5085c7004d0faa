"""The operators of the compact latent cache, as cases to time: appending
latents with the position rotation applied on the way (into the bf16 cache or
into a cache held in 8 bits), mixed-step attention over the 8-bit cache, and
mixed-step attention through a sliding window with a few first tokens that stay
visible.

Shapes are those of the served model's absorbed latent attention: 16 query heads
over one cached 576-dim latent per token (512 compressed + 64 rope dims), value =
the first 512 dims.  A case is a dict of plain values: `kind` (see run()), the
request lengths (a seeded list of decode contexts and a text of prefix:length
chunks), the page size, the output type, and window / sinks (0: every earlier
key is visible).  The lengths belong to the case, the values and page tables to
the seed: a serving step calls each operator once per layer with the same
lengths.

The 8-bit cache.  A key is held as 576 e4m3 values; every block of 16 tokens of
a page has two scales, powers of two stored as bf16, one for the 512 compressed
dims and one for the 64 rope dims.  Appending gives a block the smallest scale
that holds the largest magnitude of the tokens it writes there (448 is the
largest e4m3 value; non-finite values are stored as NaN and do not count).  A
block that already holds earlier tokens of the request keeps its scale if that is
larger; otherwise the earlier tokens are rounded again to the new scale.
"""
import math

import numpy as np
import torch

own = False

HEADS, DQK, DV, ROPE = 16, 576, 512, 64
BLOCK = 16  # tokens per pair of scales
BASE = 10000.0
SCALE = float(np.float32(1.0 / math.sqrt(192.0)))
E_MIN, E_MAX = -100, 120


def _case(name, kind, decodes, lo, hi, chunks, *, median=0.0, sigma=0.0, lens=0, page=64, out="f32", window=0, sinks=0):
    """median 0: decode contexts uniform in [lo, hi]; else lognormal, clipped to it."""
    return dict(name=name, kind=kind, decodes=decodes, median=float(median), sigma=float(sigma), lo=lo, hi=hi, lens=lens,
                chunks=chunks, page=page, out=out, window=window, sinks=sinks)


def listed():
    return [
        # a nearly idle decode node writes one token for each of four requests: latency alone
        _case("append rotated x4", "append", 4, 842, 3569, ""),
        # one layer of the headline step: 64 decode tokens and four 1024-token chunks
        _case("append rotated 64 + 4 x 1024", "append", 64, 1, 32768, "0:1024,1024:1024,3072:1024,8192:1024", median=4096, sigma=1.0, lens=4),
        # the largest decode batch writes one token per request into 8 bits: most land in a block with earlier tokens
        _case("append8 x256", "append8", 256, 512, 16384, "", lens=3),
        # a busy node with a long prompt's later chunk, at a prefix inside a block, into 8 bits
        _case("append8 128 + 2048 at 6149", "append8", 128, 16, 32768, "6149:2048", median=2048, sigma=1.2, lens=2),
        # a nearly idle node's attention over the 8-bit cache: latency and launches count
        _case("attn8 decode x4", "attn8", 4, 842, 3569, ""),
        # the largest decode batch over the 8-bit cache: bound by memory
        _case("attn8 decode x256", "attn8", 256, 512, 16384, "", lens=3),
        # a busy node with a long prompt's later chunk over the 8-bit cache: matrix-bound
        _case("attn8 128 + 2048 at 6144, bf16", "attn8", 128, 16, 32768, "6144:2048", median=2048, sigma=1.2, lens=2, out="bf16"),
        # a whole small step on the 8-bit cache (append, then attention): ragged chunks at unaligned prefixes, small pages
        _case("step8 ragged, page 16, bf16", "step8", 37, 1, 3001, "0:2,517:131,1999:333,60:601", page=16, lens=5, out="bf16"),
        # a large decode batch of long contexts through a window: what is read no longer grows with the context
        _case("window 4096 decode x256", "window", 256, 512, 32768, "", lens=8, window=4096, sinks=4),
        # the headline step's lengths through a short window with a page of sinks: chunk rows see a band
        _case("window 1024, 64 + 4 x 1024, bf16", "window", 64, 1, 32768, "0:1024,1024:1024,3072:1024,8192:1024", median=4096, sigma=1.0, lens=4,
              out="bf16", window=1024, sinks=64),
        # a lightly loaded node's first chunk: step on the 8-bit cache through an odd window, no sinks
        _case("step8 window 513, 32 + 512, bf16", "step8", 32, 16, 8192, "0:512", median=1024, sigma=1.0, lens=1, page=32, out="bf16", window=513),
    ]


def draw(rng):
    """A call of the same ranges: 1 to 256 decode requests of up to 32768 keys,
    up to four chunks of 2 to 2048 rows, windows of 1 to 8192 keys, up to 256 sinks."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        kind = rng.choice(["append", "append8", "attn8", "attn8", "step8", "window", "window"])
        decodes = log(1, 256)
        chunks = ["%d:%d" % (rng.choice([0, rng.randint(1, 8192)]), log(2, 2048)) for _ in range(rng.choice([0, 1, 1, 2, 3, 4]))]
        median, hi = (0, log(64, 16384)) if rng.random() < 0.5 else (log(64, 8192), 32768)
        band = kind == "window" or (kind in ("attn8", "step8") and rng.random() < 0.4)
        c = _case("", kind, decodes, rng.randint(1, 64), hi, ",".join(chunks), median=median, sigma=rng.choice([0.5, 1.0, 1.2]),
                  lens=rng.randrange(1 << 20), page=rng.choice([16, 32, 64, 64, 128]),
                  out="bf16" if chunks else rng.choice(["f32", "bf16"]), window=log(1, 8192) if band else 0,
                  sinks=rng.choice([0, 1, 4, log(1, 256)]) if band else 0)
        del c["name"]
        w, size = work(c), sum(_lengths(c)[0])
        if w["bytes"] <= 1.25e9 and w["flops"] <= 4.9e11 and size <= 4_200_000:
            return c


def _lengths(case):
    """(prefix, new rows) of every request: decodes, then chunks."""
    rng = np.random.default_rng(case["lens"])
    n, lo, hi = case["decodes"], case["lo"], case["hi"]
    if case["median"]:
        ctx = np.clip(np.rint(case["median"] * np.exp(case["sigma"] * rng.standard_normal(n))), lo, hi).astype(np.int64)
    else:
        ctx = rng.integers(lo, hi, n, endpoint=True)
    chunks = [tuple(int(x) for x in t.split(":")) for t in case["chunks"].split(",") if t]
    return [int(x) - 1 for x in ctx] + [p for p, _ in chunks], [1] * n + [c for _, c in chunks]


# ------------------------------------------------------------------ inputs
def _latents(gen, n):
    """n latents as they reach the cache: a gain per compressed dim, rope dims of a larger spread."""
    g = torch.Generator(device="cuda").manual_seed(11)
    gain = torch.exp(0.3 * torch.randn(DQK, device="cuda", generator=g))
    gain[DV:] *= 3.0
    return (torch.randn((n, DQK), device="cuda", generator=gen) * gain).to(torch.bfloat16)


def _block_exponent(amax):
    """Smallest E with amax 2^-E <= 448, within the range a cache holds."""
    m, e = torch.frexp(amax)
    return torch.where(m <= 0.875, e - 9, e - 8).clamp(E_MIN, E_MAX)


def _filled8(gen, slots):
    """An 8-bit cache of `slots` tokens (a multiple of 16): values and scales."""
    data = torch.empty((slots, DQK), dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty((slots // BLOCK, 2), dtype=torch.bfloat16, device="cuda")
    step = 1 << 18
    for i in range(0, slots, step):
        n = min(step, slots - i)
        x = _latents(gen, n).float().reshape(-1, BLOCK, DQK)
        a = x.abs()
        e = _block_exponent(torch.stack((a[:, :, :DV].amax(dim=(1, 2)), a[:, :, DV:].amax(dim=(1, 2))), dim=1))
        s = torch.exp2(e.float())
        x[:, :, :DV] /= s[:, :1, None]
        x[:, :, DV:] /= s[:, 1:, None]
        data[i:i + n] = x.reshape(-1, DQK).to(torch.float8_e4m3fn)
        scales[i // BLOCK:(i + n) // BLOCK] = s.to(torch.bfloat16)
    return data, scales


def prepare(case, seed):
    prefix, rows = _lengths(case)
    P, kind = case["page"], case["kind"]
    need = [-(-(p + c) // P) for p, c in zip(prefix, rows)]
    pages = int(math.ceil(1.125 * sum(need)))
    perm = np.random.default_rng([seed, 7]).permutation(pages).astype(np.int32)
    table, at = np.full((len(rows), max(need)), -1, dtype=np.int32), 0
    for r, n in enumerate(need):
        table[r, :n] = perm[at:at + n]
        at += n
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T = sum(rows)
    s = {"kind": kind, "prefix": prefix, "rows": rows, "page": P, "window": case["window"], "sinks": case["sinks"],
         "table": torch.from_numpy(table).cuda()}
    if kind in ("append", "window"):
        s["cache"] = _latents(gen, pages * P).reshape(pages, P, DQK)
    else:
        data, scales = _filled8(gen, pages * P)
        s["data"], s["scales"] = data.reshape(pages, P, DQK), scales.reshape(pages, P // BLOCK, 2)
    if kind in ("append", "append8", "step8"):
        s["new"] = _latents(gen, T)
    if kind in ("attn8", "step8", "window"):
        s["q"] = torch.randn((T, HEADS, DQK), dtype=torch.bfloat16, device="cuda", generator=gen)
        s["out"] = torch.empty((T, HEADS, DV), dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16, device="cuda")
        s["lse"] = torch.empty((T, HEADS), dtype=torch.float32, device="cuda")
    if own:  # the batch handle, cache handle and workspace that a program keeps for its steps
        import paper_2607_02043_amd as mla
        s["batch"] = mla.DeviceBatch(rows, prefix, table, P, pages)
        win = (case["window"], case["sinks"]) if case["window"] else None
        if "data" in s:
            s["cache8"] = mla.LatentCache8(data=s["data"].view(torch.uint8), scales=s["scales"])
        if kind in ("attn8", "step8"):
            s["ws"] = mla.workspace_for_cache8(s["batch"], window=win)
        elif kind == "window":
            s["ws"] = mla.workspace_for_window(s["batch"], win)
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2607_02043_amd as mla
    kind, b = s["kind"], s["batch"]
    if kind == "append":
        mla.append_latent_kv_rope(b, s["new"], BASE, s["cache"])
        return {"cache": s["cache"]}
    if kind == "window":
        mla.mixed_step_attn_window(b, s["q"], s["cache"], (s["window"], s["sinks"]), SCALE, s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    got = {}
    if kind in ("append8", "step8"):
        mla.append_latent_kv8(b, s["new"], s["cache8"], rope_base=BASE)
        got = {"data": s["data"], "scales": s["scales"]}
    if kind in ("attn8", "step8"):
        win = (s["window"], s["sinks"]) if s["window"] else None
        mla.mixed_step_attn8(b, s["q"], s["cache8"], SCALE, s["out"], s["lse"], s["ws"], window=win)
        got |= {"out": s["out"], "lse": s["lse"]}
    return got


def _run_plain(s):
    kind, got = s["kind"], {}
    if kind == "append":
        req, pos = _rows_of(s)
        s["cache"].view(-1, DQK)[_slots(s, req, pos)] = _rotated(s["new"], pos).to(torch.bfloat16)
        return {"cache": s["cache"]}
    if kind in ("append8", "step8"):
        _plain_append8(s)
        got = {"data": s["data"], "scales": s["scales"]}
    if kind in ("attn8", "step8", "window"):
        _plain_attention(s)
        got |= {"out": s["out"], "lse": s["lse"]}
    return got


def _rows_of(s):
    """Request and position of every new row."""
    c = torch.tensor(s["rows"], device="cuda")
    p = torch.tensor(s["prefix"], device="cuda")
    req = torch.repeat_interleave(torch.arange(len(s["rows"]), device="cuda"), c)
    return req, p[req] + torch.arange(req.numel(), device="cuda") - (torch.cumsum(c, 0) - c)[req]


def _slots(s, req, pos):
    """Pool slots of the tokens at `pos` of requests `req`."""
    return s["table"].long()[req, pos // s["page"]] * s["page"] + pos % s["page"]


def _rotated(new, pos):
    """Rope dims rotated, pairs (2i, 2i + 1) by pos base^(-2i / 64): angles in 64 bits, the rest in 32."""
    x = new.float()
    i = torch.arange(ROPE // 2, dtype=torch.float64, device="cuda")
    ang = pos.double()[:, None] * BASE ** (-2.0 * i / ROPE)
    c, sn = torch.cos(ang).float(), torch.sin(ang).float()
    x0, x1 = x[:, DV::2], x[:, DV + 1::2]
    return torch.cat((x[:, :DV], torch.stack((x0 * c - x1 * sn, x0 * sn + x1 * c), dim=2).flatten(1)), dim=1)


def _plain_append8(s):
    req, pos = _rows_of(s)
    x, slot = _rotated(s["new"], pos), _slots(s, req, pos)
    data, scales = s["data"].view(-1, DQK), s["scales"].view(-1, 2)
    fine = torch.where(torch.isfinite(x), x.abs(), 0.0)
    amax = torch.zeros((scales.shape[0], 2), device="cuda")
    blk = slot // BLOCK
    amax.scatter_reduce_(0, blk[:, None].expand(-1, 2), torch.stack((fine[:, :DV].amax(1), fine[:, DV:].amax(1)), dim=1), "amax")
    e = _block_exponent(amax)
    # blocks that hold earlier tokens of their request: one at most for each request
    p = torch.tensor(s["prefix"], device="cuda")
    r = torch.nonzero(p % BLOCK != 0).flatten()
    first = p[r] // BLOCK * BLOCK
    held = _slots(s, r, first) // BLOCK
    old = torch.frexp(scales[held].float())[1] - 1
    e[held] = torch.maximum(e[held], old)
    at = (held[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")).flatten()
    earlier = (torch.arange(BLOCK, device="cuda")[None, :] < (p[r] - first)[:, None]).flatten()
    at = at[earlier]
    down = torch.exp2((old - e[held]).float())[:, None, :].expand(-1, BLOCK, 2).reshape(-1, 2)[earlier]
    v = data[at].float()
    data[at] = torch.cat((v[:, :DV] * down[:, :1], v[:, DV:] * down[:, 1:]), dim=1).to(torch.float8_e4m3fn)
    sc = torch.exp2(e[blk].float())
    y = torch.cat((x[:, :DV] / sc[:, :1], x[:, DV:] / sc[:, 1:]), dim=1)
    data[slot] = torch.where(torch.isfinite(y), y, math.nan).to(torch.float8_e4m3fn)
    scales[blk] = sc.to(torch.bfloat16)


def _keys(s, slot):
    """Cached latents of these slots, 32 bits."""
    if "cache" in s:
        return s["cache"].view(-1, DQK)[slot].float()
    sc = s["scales"].view(-1, 2)[slot // BLOCK].float()
    v = s["data"].view(-1, DQK)[slot].float()
    v[..., :DV] *= sc[..., :1]
    v[..., DV:] *= sc[..., 1:]
    return v


def _hidden(s, key, pos):
    """Keys that a row at `pos` does not see."""
    away = key > pos
    if s["window"]:
        away = away | ((key <= pos - s["window"]) & (key >= s["sinks"]))
    return away


def _softmax_v(x, keys):
    """x scores [.., rows, keys]: weighted values and the log of the sum."""
    l = torch.logsumexp(x, dim=-1)
    return torch.exp(x - l[..., None]) @ keys[..., :DV], l


def _plain_attention(s):
    n = sum(1 for c in s["rows"] if c == 1)  # the decode requests come first
    if n:
        p = torch.tensor(s["prefix"][:n], device="cuda")
        key = torch.arange(max(s["prefix"][:n]) + 1, device="cuda")[None, :].expand(n, -1)
        keys = _keys(s, _slots(s, torch.arange(n, device="cuda")[:, None], torch.minimum(key, p[:, None])))
        x = torch.bmm(s["q"][:n].float(), keys.transpose(1, 2)) * SCALE
        x.masked_fill_(_hidden(s, key, p[:, None])[:, None, :], -math.inf)
        o, l = _softmax_v(x, keys)
        s["out"][:n], s["lse"][:n] = o.to(s["out"].dtype), l
    row = n
    for r in range(n, len(s["rows"])):
        p, c = s["prefix"][r], s["rows"][r]
        key = torch.arange(p + c, device="cuda")
        keys = _keys(s, _slots(s, torch.full_like(key, r), key))
        x = (s["q"][row:row + c].float().reshape(c * HEADS, DQK) @ keys.T).reshape(c, HEADS, p + c) * SCALE
        x.masked_fill_(_hidden(s, key[None, :], p + torch.arange(c, device="cuda")[:, None])[:, None, :], -math.inf)
        o, l = _softmax_v(x.reshape(c * HEADS, p + c), keys)
        s["out"][row:row + c], s["lse"][row:row + c] = o.reshape(c, HEADS, DV).to(s["out"].dtype), l.reshape(c, HEADS)
        row += c


# ------------------------------------------------------------------ work
def _visible(case, p, c):
    """(query-key pairs, distinct cached keys read) of a request."""
    w, k = case["window"], case["sinks"]
    pos = np.arange(p, p + c, dtype=np.int64)
    if not w:
        return int((pos + 1).sum()), p + c
    first = np.maximum(pos - w + 1, 0)
    pairs = int((pos + 1 - first + np.minimum(first, k)).sum())
    lo = max(p - w + 1, 0)
    return pairs, p + c - lo + min(lo, k)


def work(case):
    prefix, rows = _lengths(case)
    kind, T, R = case["kind"], sum(rows), len(rows)
    key = 2 * DQK if kind in ("append", "window") else DQK + 4 / BLOCK
    out = {"bytes": 12.0 * R, "flops": 0.0}
    if kind in ("append", "append8", "step8"):
        # new latents read, keys written, page ids; a rotation of 32 pairs and, in 8 bits, two operations a value
        out["bytes"] += 2 * DQK * T + key * T + 4 * sum(-(-c // case["page"]) for c in rows)
        out["flops"] += T * (6 * ROPE // 2 + (0 if kind == "append" else 2 * DQK))
    if kind in ("attn8", "step8", "window"):
        seen = [_visible(case, p, c) for p, c in zip(prefix, rows)]
        keys = sum(k for _, k in seen)
        out["bytes"] += key * keys + 4 * keys / case["page"] + 2 * HEADS * DQK * T + HEADS * T * (DV * (4 if case["out"] == "f32" else 2) + 4)
        out["flops"] += 2.0 * HEADS * (DQK + DV) * sum(n for n, _ in seen)
    return out


# ------------------------------------------------------------------ in 64 bits
def _e4m3(v):
    """Nearest e4m3 value, ties to even: steps of 2^(e - 3) from 2^e on, 2^-9 below 2^-6."""
    m, e = torch.frexp(v)  # |v| = m 2^e, 0.5 <= m < 1
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return torch.where(torch.isfinite(v), torch.round(v / step) * step, math.nan)


def _exact_append8(s):
    data, scales = s["data"].double().reshape(-1, DQK), s["scales"].double().reshape(-1, 2)
    P, row, parts = s["page"], 0, ((0, DV), (DV, DQK))
    table = s["table"].cpu().numpy()
    for r, (p, c) in enumerate(zip(s["prefix"], s["rows"])):
        t = torch.arange(p, p + c, device="cuda")
        x = _exact_rope(s["new"][row:row + c].double(), t)
        row += c
        # all blocks of the request at once, tokens before p and behind the last one as zeros
        b0, b1 = p // BLOCK, (p + c - 1) // BLOCK + 1
        whole = torch.zeros(((b1 - b0) * BLOCK, DQK), dtype=torch.float64, device="cuda")
        whole[p - b0 * BLOCK:p - b0 * BLOCK + c] = x
        g = torch.arange(b0 * BLOCK, b1 * BLOCK, device="cuda")
        slot = torch.from_numpy(table[r].astype(np.int64)).cuda()[g // P] * P + g % P
        blk = slot.reshape(-1, BLOCK)[:, 0] // BLOCK
        for k, (d0, d1) in enumerate(parts):
            part = whole[:, d0:d1].reshape(-1, BLOCK, d1 - d0)
            a = torch.where(torch.isfinite(part), part.abs(), 0.0).amax(dim=(1, 2))
            e = torch.ceil(torch.log2(a / 448.0)).clamp(E_MIN, E_MAX)  # (log2 0 = -inf)
            e = torch.where(a * torch.exp2(-e) > 448.0, e + 1, torch.where((a * torch.exp2(1 - e) <= 448.0) & (e > E_MIN), e - 1, e))
            if p % BLOCK:
                was = torch.log2(scales[blk[0], k])
                e[0] = torch.maximum(e[0], was)
                old = slot[:p - b0 * BLOCK]
                data[old, d0:d1] = _e4m3(data[old, d0:d1] * torch.exp2(was - e[0]))
            sc = torch.exp2(e)
            n = slice(p - b0 * BLOCK, p - b0 * BLOCK + c)
            data[slot[n], d0:d1] = _e4m3((part / sc[:, None, None]).reshape(-1, d1 - d0)[n])
            scales[blk, k] = sc
    return data.reshape(s["data"].shape), scales.reshape(s["scales"].shape)


def _exact_rope(x, pos):
    """x 64 bits [rows][576], rotated as complex numbers."""
    f = BASE ** (-torch.arange(0, ROPE, 2, dtype=torch.float64, device="cuda") / ROPE)
    z = torch.view_as_complex(x[:, DV:].reshape(-1, ROPE // 2, 2).contiguous())
    z = z * torch.polar(torch.ones_like(f)[None, :], pos.double()[:, None] * f)
    return torch.cat((x[:, :DV], torch.view_as_real(z).reshape(-1, ROPE)), dim=1)


def exact(case, seed):
    s = prepare(case, seed)
    prefix, rows, P, kind, got = s["prefix"], s["rows"], s["page"], s["kind"], {}
    first = np.concatenate(([0], np.cumsum(rows)))
    table = s["table"].cpu().numpy().astype(np.int64)
    if kind == "append":
        cache = s["cache"].double().reshape(-1, DQK)
        for r, (p, c) in enumerate(zip(prefix, rows)):
            t = np.arange(p, p + c)
            slot = torch.from_numpy(table[r, t // P] * P + t % P).cuda()
            cache[slot] = _exact_rope(s["new"][first[r]:first[r + 1]].double(), torch.from_numpy(t).cuda())
        return {"cache": cache.reshape(s["cache"].shape)}
    if kind in ("append8", "step8"):
        data, scales = _exact_append8(s)
        got = {"data": data, "scales": scales}
        if kind == "append8":
            return got
    elif kind == "attn8":
        data, scales = s["data"], s["scales"]
    out = torch.empty((first[-1], HEADS, DV), dtype=torch.float64, device="cuda")
    lse = torch.empty((first[-1], HEADS), dtype=torch.float64, device="cuda")
    for r, (p, c) in enumerate(zip(prefix, rows)):
        t = np.arange(p + c)
        slot = torch.from_numpy(table[r, t // P] * P + t % P).cuda()
        if kind == "window":
            keys = s["cache"].reshape(-1, DQK)[slot].double()
        else:
            sc = scales.reshape(-1, 2)[slot // BLOCK].double()
            keys = data.reshape(-1, DQK)[slot].double()
            keys = torch.cat((keys[:, :DV] * sc[:, :1], keys[:, DV:] * sc[:, 1:]), dim=1)
        step = max(1, (1 << 26) // (HEADS * (p + c)))
        for i in range(0, c, step):
            n = min(step, c - i)
            at = slice(first[r] + i, first[r] + i + n)
            row, key = p + i + torch.arange(n, device="cuda")[:, None], torch.arange(p + c, device="cuda")[None, :]
            seen = key <= row
            if s["window"]:
                seen = seen & ((row - key < s["window"]) | (key < s["sinks"]))
            x = torch.matmul(s["q"][at].double().reshape(n * HEADS, DQK), keys.T).reshape(n, HEADS, p + c) * SCALE
            m = torch.where(seen[:, None, :], x, -math.inf).amax(dim=2, keepdim=True)
            e = torch.where(seen[:, None, :], torch.exp(x - m), 0.0)
            z = e.sum(dim=2)
            lse[at] = m[:, :, 0] + torch.log(z)
            out[at] = torch.matmul(e.reshape(n * HEADS, p + c), keys[:, :DV]).reshape(n, HEADS, DV) / z[:, :, None]
    return got | {"out": out, "lse": lse}
