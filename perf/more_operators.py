"""The feed-forward half of a layer, as cases to time: a gated feed-forward block
with bf16 weights, products with 4-bit weights in groups that share a scale, and
the feed-forward block with such weights.

x is bf16 [rows][hidden].  The block computes
    g = x Wg^T,  u = x Wu^T,  h = g / (1 + exp(-g)) * u,  out = h Wd^T
with Wg, Wu [inner][hidden] and Wd [hidden][inner]; a product with 4-bit weights
computes out = x W^T with W [cols][hidden].

4-bit weights.  A code has a sign bit (8) and a magnitude out of 0, 0.5, 1, 1.5,
2, 3, 4, 6; each 32 neighbouring weights of a row share one scale byte b, which
stands for 2^(b - 127).  Codes are packed two a byte, the even one in the low half:
codes [cols][in / 2], scales [cols][in / 32].

The widths are the served model's hidden width (2048) with generic inner widths
and output widths; the row counts are those of a decode node's steps: its
decodes, alone or with a prompt's chunk beside them.
"""
import math

import torch

own = False

GROUP = 32
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, kind, rows, hidden, inner, out):
    """inner: the inner width of a feed-forward block, the output width of a product."""
    return dict(name=name, kind=kind, rows=rows, hidden=hidden, inner=inner, out=out)


def listed():
    return [
        # one request on an idle node: a square projection of its token, latency alone
        _case("linear4 x1, 2048 square", "linear4", 1, 2048, 2048, "bf16"),
        # a small decode batch's logits over a large vocabulary: bound by reading the weights
        _case("linear4 x32, 102400 wide", "linear4", 32, 2048, 102400, "f32"),
        # a decode batch beside a short prompt's tail, an output width that no tile divides
        _case("linear4 x173, 5000 wide", "linear4", 173, 2048, 5000, "f32"),
        # the headline step's 64 decodes and four 1024-token chunks: bound by the products
        _case("linear4 x4160, 8192 wide", "linear4", 4160, 2048, 8192, "bf16"),
        # a nearly idle decode node, a narrow block: latency and launches count
        _case("ffn x4, 1408", "ffn", 4, 2048, 1408, "bf16"),
        # a decode batch, a wide block: bound by reading the weights
        _case("ffn x64, 10944", "ffn", 64, 2048, 10944, "f32"),
        # a lightly loaded node with a prompt's first chunk, the inner width of an eighth share
        _case("ffn x544, 1368", "ffn", 544, 2048, 1368, "bf16"),
        # the headline step: bound by the products
        _case("ffn x4160, 10944", "ffn", 4160, 2048, 10944, "bf16"),
        # one request on an idle node, a wide block in 4 bits
        _case("ffn4 x1, 10944", "ffn4", 1, 2048, 10944, "bf16"),
        # a mid-sized decode batch in 4 bits, odd rows
        _case("ffn4 x37, 5504", "ffn4", 37, 2048, 5504, "f32"),
        # the largest decode batch in 4 bits
        _case("ffn4 x256, 10944", "ffn4", 256, 2048, 10944, "bf16"),
        # a busy node with a long prompt's chunk, in 4 bits
        _case("ffn4 x2176, 5504", "ffn4", 2176, 2048, 5504, "bf16"),
    ]


def draw(rng):
    """A call of the same ranges: 1 to 4160 rows, hidden widths 256 to 4096, inner
    widths 256 to 10944, output widths 64 to 102400."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        kind = rng.choice(["linear4", "ffn", "ffn4"])
        hidden = rng.choice([2048, 2048, 32 * rng.randint(8, 128)])
        step = 8 if kind != "ffn4" else GROUP
        inner = log(64, 102400) if kind == "linear4" else log(256, 10944)
        c = _case("", kind, log(1, 4160), hidden, max(step, inner // step * step), rng.choice(["bf16", "bf16", "f32"]))
        del c["name"]
        w = work(c)
        if w["bytes"] <= 1.65e8 and w["flops"] <= 5.5e11:
            return c


# ------------------------------------------------------------------ inputs
def _weights4(gen, rows, cols):
    """Random 4-bit weights of variance 1 / cols: each group of 32 under the smallest scale
    with which its largest magnitude is at most 6."""
    codes = torch.empty((rows, cols // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((rows, cols // GROUP), dtype=torch.uint8, device="cuda")
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")
    step = max(1, (1 << 25) // cols)
    for i in range(0, rows, step):
        n = min(step, rows - i)
        w = torch.randn((n, cols // GROUP, GROUP), device="cuda", generator=gen) / math.sqrt(cols)
        e = torch.ceil(torch.log2(w.abs().amax(dim=2).clamp(min=1e-30) / 6.0))
        c = torch.bucketize(w.abs() * torch.exp2(-e)[:, :, None], edges, out_int32=True) + 8 * (w < 0)
        c = c.reshape(n, cols // 2, 2).to(torch.uint8)
        codes[i:i + n] = c[:, :, 0] + 16 * c[:, :, 1]
        scales[i:i + n] = (e + 127.0).to(torch.uint8)
    return codes, scales


def _weights(gen, rows, cols):
    return (torch.randn((rows, cols), device="cuda", generator=gen) / math.sqrt(cols)).to(torch.bfloat16)


def prepare(case, seed):
    kind, T, H, N = case["kind"], case["rows"], case["hidden"], case["inner"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    # rows behind a norm: a gain per dim
    gain = torch.exp(0.3 * torch.randn(H, device="cuda", generator=gen))
    s = {"kind": kind, "x": (torch.randn((T, H), device="cuda", generator=gen) * gain).to(torch.bfloat16)}
    dtype = torch.float32 if case["out"] == "f32" else torch.bfloat16
    make = _weights if kind == "ffn" else _weights4
    if kind == "linear4":
        s["w"] = make(gen, N, H)
    else:
        s["gate"], s["up"], s["down"] = make(gen, N, H), make(gen, N, H), make(gen, H, N)
    s["out"] = torch.empty((T, N if kind == "linear4" else H), dtype=dtype, device="cuda")
    if own:  # the weights' handle and the workspace that a program keeps for its steps
        import paper_2607_02043_amd as mla
        if kind == "linear4":
            s["weights"] = mla.Weights4(*s["w"])
            s["ws"] = mla.workspace_for_linear4(T, s["weights"])
        else:
            w = [s[k] if kind == "ffn" else mla.Weights4(*s[k]) for k in ("gate", "up", "down")]
            s["weights"] = mla.FfnWeights(*w)
            s["ws"] = mla.workspace_for_ffn(T, s["weights"])
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2607_02043_amd as mla
    if s["kind"] == "linear4":
        mla.linear4(s["x"], s["weights"], s["out"], s["ws"])
    else:
        mla.gated_ffn(s["x"], s["weights"], s["out"], s["ws"])
    return s["out"]


def _values(w):
    """Weights as 32-bit numbers."""
    if isinstance(w, torch.Tensor):
        return w.float()
    codes, scales = w
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device="cuda")
    pair = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), dim=2)
    return (pair.reshape(codes.shape[0], -1, GROUP) * torch.exp2(scales.float() - 127.0)[:, :, None]).reshape(codes.shape[0], -1)


def _run_plain(s):
    x = s["x"].float()
    if s["kind"] == "linear4":
        y = x @ _values(s["w"]).T
    else:
        g, u = x @ _values(s["gate"]).T, x @ _values(s["up"]).T
        y = (g / (1.0 + torch.exp(-g)) * u) @ _values(s["down"]).T
    s["out"].copy_(y)
    return s["out"]


# ------------------------------------------------------------------ work
def work(case):
    kind, T, H, N = case["kind"], case["rows"], case["hidden"], case["inner"]
    n = N * H * (1 if kind == "linear4" else 3)  # weights
    wide = N if kind == "linear4" else H
    return {"bytes": n * (2.0 if kind == "ffn" else 0.5 + 1.0 / GROUP) + 2.0 * T * H + T * wide * (4.0 if case["out"] == "f32" else 2.0),
            "flops": 2.0 * T * n}


# ------------------------------------------------------------------ in 64 bits
def _exact_weights(w):
    if isinstance(w, torch.Tensor):
        return w.double()
    codes, scales = (t.long() for t in w)
    c = torch.empty((codes.shape[0], codes.shape[1] * 2), dtype=torch.int64, device="cuda")
    c[:, 0::2], c[:, 1::2] = codes % 16, codes // 16
    m, e = c % 2, c // 2 % 4  # one mantissa bit, two exponent bits of bias 1, e = 0: halves
    v = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * torch.exp2((e - 1).double()))
    v = torch.where(c >= 8, -v, v)
    return v * torch.exp2((scales - 127).double()).repeat_interleave(GROUP, dim=1)


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    if s["kind"] == "linear4":
        step = 8192
        parts = [torch.matmul(x, _exact_weights([t[i:i + step] for t in s["w"]]).mT) for i in range(0, case["inner"], step)]
        return torch.cat(parts, dim=1)
    g = torch.matmul(x, _exact_weights(s["gate"]).mT)
    h = g * torch.sigmoid(g)
    h *= torch.matmul(x, _exact_weights(s["up"]).mT)
    return torch.matmul(h, _exact_weights(s["down"]).mT)
