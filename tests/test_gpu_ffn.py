"""The feed-forward operators against their definition in 64 bits (needs an MI355X)."""
import math

import numpy as np
import pytest
import torch

import paper_2607_02043_amd as mla
from ffn_cases import Matrix, assert_within, bf16, block, ffn, linear4, rows
from harness import log
from oracle import ffn_oracle as O

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _name(v):
    return {F32: "f32", BF16: "bf16"}.get(v)


# rows: one, inside and at the edges of 16-row blocks and of every tile height, chunks
ROWS = (1, 2, 4, 15, 16, 17, 31, 33, 48, 49, 64, 65, 100, 128, 129, 250, 257, 300, 515)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=_name)
@pytest.mark.parametrize("T", ROWS)
def test_linear4_rows(T, dtype):
    log(f"[gpu] linear4 rows {T} {dtype}")
    x, w = rows(1, T, 352), Matrix(2, 200, 352, True)
    assert_within(linear4(x, w, dtype), *O.linear(x.double().numpy(), w.values), dtype, f"{T} rows")


# widths: one group and odd numbers of them, ends inside a stage and a slice; outputs from 8 columns on
FEW = (1, 5, 40, 70, 300)
LINEAR_SIZES = [(32, 8), (64, 24), (96, 40), (160, 1000), (416, 136), (2048, 72), (1376, 264), (10944, 16)]


@pytest.mark.parametrize("T", FEW)
@pytest.mark.parametrize("k,n", LINEAR_SIZES)
def test_linear4_sizes(T, k, n):
    log(f"[gpu] linear4 {T} x {k} -> {n}")
    x, w = rows(3, T, k), Matrix(4, n, k, True)
    assert_within(linear4(x, w, F32), *O.linear(x.double().numpy(), w.values), F32, f"{T} x {k} -> {n}")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=_name)
@pytest.mark.parametrize("four", [False, True], ids=["bf16w", "mx4"])
@pytest.mark.parametrize("T", ROWS)
def test_ffn_rows(T, four, dtype):
    log(f"[gpu] ffn rows {T} {four} {dtype}")
    x, mats = rows(5, T, 288), block(6, 288, 416, four)
    ref = O.ffn(x.double().numpy(), *(m.values for m in mats), 3 if dtype == F32 else 1)
    assert_within(ffn(x, mats, dtype), *ref, dtype, f"{T} rows")


SIZES = [(8, 8), (24, 40), (40, 8), (72, 1368), (2048, 24), (1000, 200)]
SIZES4 = [(32, 32), (96, 32), (32, 160), (2048, 96), (160, 1376), (1024, 224)]


@pytest.mark.parametrize("T", FEW)
@pytest.mark.parametrize("four,hidden,inner", [(False, *s) for s in SIZES] + [(True, *s) for s in SIZES4])
def test_ffn_sizes(T, four, hidden, inner):
    log(f"[gpu] ffn {T} x {hidden} x {inner} {four}")
    x, mats = rows(7, T, hidden), block(8, hidden, inner, four)
    ref = O.ffn(x.double().numpy(), *(m.values for m in mats), 3)
    assert_within(ffn(x, mats, F32), *ref, F32, f"{T} x {hidden} x {inner}")


# (0 product with 4-bit weights, 1 block in bf16, 2 block in 4 bits; rows; in or hidden; out or inner; fp32 output): calls
# that between them choose every kernel, whole and in parts, in every product that it takes, and rows left to a second launch
EVERY_KERNEL = [
    (0, 21, 2944, 16752, 0), (0, 2169, 96, 40, 0), (0, 2207, 2656, 40, 0), (0, 2249, 5344, 952, 1), (0, 2759, 3744, 72, 1),
    (0, 2775, 2720, 40, 0), (0, 2912, 6784, 752, 0), (0, 3258, 160, 200, 1), (0, 4180, 2080, 32, 0), (0, 4253, 3968, 8, 0),
    (0, 4447, 192, 80, 0), (0, 4461, 160, 8, 1), (0, 4479, 2304, 8, 1), (1, 2, 2056, 8, 0), (1, 4, 8, 328, 1), (1, 10, 8, 1056, 0),
    (1, 703, 24, 2440, 1), (1, 737, 3184, 16, 0), (1, 952, 64, 2376, 0), (1, 1040, 24, 2680, 0), (1, 1048, 112, 200, 1),
    (1, 1361, 3152, 728, 1), (1, 1552, 64, 1344, 0), (1, 1636, 1088, 40, 0), (1, 1781, 72, 520, 1), (1, 1925, 2128, 8, 1),
    (1, 2121, 1128, 24, 0), (1, 2378, 40, 520, 1), (1, 2503, 904, 4200, 0), (1, 2552, 3160, 72, 1), (1, 2590, 1728, 4944, 0),
    (1, 2773, 712, 1072, 1), (1, 2785, 24, 528, 0), (1, 2892, 8, 136, 0), (1, 2954, 656, 4320, 0), (1, 3265, 1240, 72, 1),
    (1, 3368, 72, 624, 1), (1, 3596, 1272, 1600, 1), (1, 3695, 1064, 72, 0), (1, 3714, 10504, 320, 0), (1, 3791, 1224, 2000, 1),
    (1, 3882, 80, 1192, 0), (1, 4173, 8, 1864, 0), (1, 4180, 16, 10728, 1), (1, 4186, 952, 5440, 0), (1, 4212, 160, 3048, 0),
    (1, 4225, 3504, 8, 0), (1, 4253, 16, 8448, 0), (1, 4256, 24, 2104, 0), (1, 4262, 24, 11160, 1), (1, 4302, 1552, 8, 1),
    (1, 4303, 4104, 208, 0), (1, 4305, 8, 200, 1), (1, 4310, 8, 1040, 1), (1, 4339, 8, 2560, 1), (1, 4355, 4560, 496, 0),
    (1, 4366, 8, 2264, 1), (1, 4387, 408, 3456, 1), (1, 4426, 3648, 96, 0), (2, 18, 32, 1568, 1), (2, 19, 8704, 3264, 1),
    (2, 21, 2080, 8704, 0), (2, 56, 416, 2304, 1), (2, 341, 128, 2080, 1), (2, 369, 3136, 32, 1), (2, 393, 2720, 32, 1),
    (2, 408, 9504, 96, 1), (2, 451, 4256, 1920, 1), (2, 480, 128, 4192, 1), (2, 677, 32, 3232, 0), (2, 684, 5184, 32, 1),
    (2, 801, 64, 7424, 0), (2, 1037, 544, 32, 0), (2, 1155, 32, 4000, 1), (2, 1238, 7584, 32, 0), (2, 1413, 7328, 128, 1),
    (2, 1420, 5440, 768, 1), (2, 1532, 96, 32, 1), (2, 1693, 2432, 160, 1), (2, 1812, 2720, 288, 1), (2, 2103, 96, 32, 1),
    (2, 2125, 64, 672, 1), (2, 2186, 2368, 32, 1), (2, 2220, 64, 800, 1), (2, 2699, 1472, 32, 0), (2, 2700, 1696, 5184, 0),
    (2, 2743, 160, 4320, 0), (2, 2935, 5312, 768, 1), (2, 3380, 1216, 800, 0), (2, 3421, 672, 2240, 1), (2, 3458, 1248, 2048, 1),
    (2, 3546, 8256, 288, 1), (2, 3737, 160, 1664, 1), (2, 4101, 3424, 256, 0), (2, 4187, 96, 32, 1), (2, 4213, 2112, 32, 1),
    (2, 4234, 32, 1088, 1), (2, 4255, 96, 864, 1), (2, 4313, 160, 96, 0), (2, 4473, 160, 32, 1),
]


@pytest.mark.parametrize("what,T,k,n,f32", EVERY_KERNEL)
def test_every_kernel(what, T, k, n, f32):
    log(f"[gpu] every kernel {what} {T} {k} {n} {f32}")
    dtype, four = (F32 if f32 else BF16), what != 1
    x = rows(31, T, k)
    # the first and last rows, those at each multiple of 128 (tiles and second launches begin there), 64 more
    edge = np.arange(0, T, 128)
    at = np.unique(np.concatenate((np.arange(min(T, 8)), np.arange(max(0, T - 8), T), edge, edge[1:] - 1, np.random.default_rng(1).integers(0, T, 64))))
    if what == 0:
        w = Matrix(32, n, k, True)
        got, ref = linear4(x, w, dtype), O.linear(x[at].double().numpy(), w.values)
    else:
        mats = block(33, k, n, four)
        got, ref = ffn(x, mats, dtype), O.ffn(x[at].double().numpy(), *(m.values for m in mats), 3 if f32 else 1)
    assert_within(got[at], *ref, dtype, f"{what} {T} x {k} x {n}")


@pytest.mark.parametrize("what,T,k,n,f32", EVERY_KERNEL)
def test_rows_keep_to_themselves(what, T, k, n, f32):
    """Rows that are not finite change no bit of the others, in every kernel."""
    log(f"[gpu] rows apart {what} {T} {k} {n} {f32}")
    dtype, four = (F32 if f32 else BF16), what != 1
    x = rows(41, T, k)
    bad = torch.from_numpy(np.unique(np.random.default_rng([T, k]).integers(0, T, 1 + T // 50)))
    y = x.clone()
    y[bad, 0], y[bad, k - 1] = math.nan, math.inf
    if what == 0:
        w = Matrix(42, n, k, True)
        one, two = linear4(x, w, dtype), linear4(y, w, dtype)
    else:
        mats = block(43, k, n, four)
        one, two = ffn(x, mats, dtype), ffn(y, mats, dtype)
    assert np.isfinite(one).all() and np.isnan(two[bad]).all()
    others = np.setdiff1d(np.arange(T), bad.numpy())
    assert np.array_equal(one[others], two[others])


@pytest.mark.parametrize("four", [False, True], ids=["bf16w", "mx4"])
def test_calls_at_once(four):
    """Calls on two streams, each with a workspace of its own, as often as they may meet."""
    mats = block(44, 2048, 1376, four)
    W, L = mla.FfnWeights(*(m.device() for m in mats)), Matrix(45, 1000, 2048, True).device()
    xs = [rows(46, T, 2048).cuda() for T in (40, 130)]
    spaces = [(mla.workspace_for_ffn(130, W), mla.workspace_for_linear4(130, L)) for _ in xs]

    def both(i, stream=None):
        outs = torch.empty((len(xs[i]), 2048), dtype=F32, device="cuda"), torch.empty((len(xs[i]), 1000), dtype=BF16, device="cuda")
        mla.gated_ffn(xs[i], W, outs[0], spaces[i][0], stream=stream)
        mla.linear4(xs[i], L, outs[1], spaces[i][1], stream=stream)
        return outs

    want = [both(0), both(1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(20):
        for i in (0, 1):
            got.append((i, both(i, streams[i])))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i, outs in got for a, b in zip(outs, want[i]))


@pytest.mark.parametrize("four", [False, True], ids=["bf16w", "mx4"])
@pytest.mark.parametrize("T", [1, 19, 64, 200, 544])
def test_ffn_real_widths(T, four):
    log(f"[gpu] ffn {T} x 2048 x 1408 {four}")
    x, mats = rows(9, T, 2048), block(10, 2048, 1408, four)
    for dtype in (F32, BF16):
        ref = O.ffn(x.double().numpy(), *(m.values for m in mats), 3 if dtype == F32 else 1)
        got = ffn(x, mats, dtype)
        assert_within(got, *ref, dtype, f"{T} rows, {dtype}")
        # in the 2-norm random signs leave of each rounding of relative 2^-8 at most that: h and out are rounded once each
        rel = np.linalg.norm(got - ref[0]) / np.linalg.norm(ref[0])
        assert rel <= (2 * 2.0 ** -8 if dtype == BF16 else 2e-5), rel


@pytest.mark.parametrize("T", [1, 3, 40, 300])
def test_scales_of_every_byte(T):
    """Scale bytes 0 .. 252 in one row each (values down to 2^-128, below the normal bf16 range), NaN for 255."""
    k, n = 64, 256
    x = torch.zeros((T, k), dtype=BF16)
    x[:, 5], x[:, 37] = 1.0, 0.0
    w = Matrix(1, n, k, True)
    w.codes[:], w.scales[:] = 0x53, 127
    w.scales[:, 0] = torch.arange(n, dtype=torch.uint8)
    got, ref = linear4(x, w, F32), w.values
    ref = x.double().numpy() @ np.where(np.isnan(ref), 0.0, np.where(np.isinf(ref), 0.0, ref)).T
    assert np.array_equal(got[:, :253], ref[:, :253]), "one product, exact"
    assert np.isnan(got[:, 255]).all()
    # 253, 254: magnitude 5 is 3 (2^127.6: finite); at 254 it is 2^128.6, infinite, and 0 x inf is NaN
    assert np.array_equal(got[:, 253], ref[:, 253]) and np.isnan(got[:, 254]).all()


@pytest.mark.parametrize("four", [False, True], ids=["bf16w", "mx4"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=_name)
@pytest.mark.parametrize("T", [3, 20, 70, 300])
def test_values_that_are_not_finite_stay_in_their_rows(T, dtype, four):
    log(f"[gpu] ffn not finite {T} {dtype} {four}")
    x, mats = rows(11, T, 96), block(12, 96, 160, four)
    clean = ffn(x, mats, dtype)
    dirty = x.clone()
    dirty[0, 95], dirty[T // 2, 0], dirty[T - 1, 17] = float("nan"), float("inf"), float("-inf")
    got = ffn(dirty, mats, dtype)
    keep = np.ones(T, dtype=bool)
    keep[[0, T // 2, T - 1]] = False
    assert np.array_equal(got[keep], clean[keep])
    assert not np.isfinite(got[~keep]).any()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=_name)
@pytest.mark.parametrize("T", [2, 40, 300])
def test_large_gates_and_infinite_h(T, dtype):
    """Gates of +-1000 saturate (silu(-1000) is 0); an h that overflows is infinite in its columns' outputs, with its sign."""
    hidden, inner = 32, 40
    x = torch.zeros((T, hidden), dtype=BF16)
    x[:, 0] = 1.0
    mats = block(1, hidden, inner, False)
    for m in mats:
        m.w[:] = 0
    gate, up, down = (m.w for m in mats)
    gate[0, 0], up[0, 0] = 1000.0, 3.0
    gate[1, 0], up[1, 0] = -1000.0, 5.0
    gate[2, 0], up[2, 0] = 1e30, 1e30
    down[0, 0] = 2.0
    down[1, 1] = 7.0
    got = ffn(x, mats, dtype)
    # the infinite h[2] meets weights of 0 in every output column
    assert np.isnan(got).all()
    down[:, 2] = 1.0
    down[5, 2] = -1.0
    got = ffn(x, mats, dtype)
    assert np.all(got[:, 5] == -np.inf) and np.all(np.delete(got, 5, axis=1) == np.inf)
    up[2, 0] = 0.0
    got = ffn(x, mats, dtype)
    # h = 3000 lies between the bf16 values 2992 and 3008: off by half a step before the output's own rounding
    assert np.all(np.abs(got[:, 0] - 6000.0) <= (0.0 if dtype == F32 else 2 * 2.0 ** -8 * 6000.0)) and not got[:, 1:].any()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=_name)
@pytest.mark.parametrize("T", [2, 40, 300, 1100])
def test_infinite_weights_of_the_down_projection(T, dtype):
    """An infinite weight makes its column infinite with the sign of h, whatever the bits of h; beside others of the same
    sign too, and an infinite h beside it."""
    hidden, inner = 128, 160
    x, mats = rows(61, T, hidden), block(62, hidden, inner, False)
    mats[2].w[7, 3] = math.inf
    mats[2].w[9, 100] = -math.inf
    assert_within(ffn(x, mats, dtype), *O.ffn(x.double().numpy(), *(m.values for m in mats), 3 if dtype == F32 else 1), dtype, "random h")
    for m in mats:
        m.w[:] = 0
    x[:] = 0
    x[:, 0] = 1.0
    gate, up, down = (m.w for m in mats)
    gate[0, 0], up[0, 0] = 1000.0, 3.0     # h = 3000: two planes and nothing behind them
    gate[1, 0], up[1, 0] = 1024.0, -2.0    # h = -2048: one
    gate[2, 0], up[2, 0] = 1e30, 1e30      # h infinite
    down[:, 2] = 1.0
    down[:2, 0], down[2:4, 1], down[4, 2] = math.inf, -math.inf, math.inf
    down[5:7, 0], down[5, 1], down[6, 1] = math.inf, -math.inf, math.inf
    down[:, 3:] = 1.0
    got = ffn(x, mats, dtype)
    assert np.all(got[:, [0, 1, 2, 3, 4, 5, 7]] == np.inf) and np.isnan(got[:, 6]).all()


@pytest.mark.parametrize("T", [2, 40, 300])
def test_infinite_4_bit_weights_of_the_down_projection(T):
    x, mats = rows(63, T, 64), block(64, 64, 96, True)
    mats[2].codes[5, 16:32], mats[2].scales[5, 1] = 0, 254
    mats[2].codes[5, 20] = 0x50  # 3 x 2^127 at k = 41 of column 5: infinite, nothing else of its group
    ref = O.ffn(x.double().numpy(), *(m.values for m in mats), 3)
    assert np.isinf(ref[0][:, 5]).all()
    assert_within(ffn(x, mats, F32), *ref, F32, f"{T} rows")


@pytest.mark.parametrize("four", [False, True], ids=["bf16w", "mx4"])
@pytest.mark.parametrize("T", [1, 50, 200, 700])
def test_same_call_same_bits_on_another_stream_and_a_larger_workspace(T, four):
    x, mats = rows(13, T, 2048).cuda(), block(14, 2048, 1408, four)
    W = mla.FfnWeights(*(m.device() for m in mats))
    ws = mla.workspace_for_ffn(T + 1000, W)
    ws[mla.MLA_FFN_COUNTER_BYTES:] = 0xA5
    outs = [torch.empty((T, 2048), dtype=F32, device="cuda") for _ in range(4)]
    mla.gated_ffn(x, W, outs[0], mla.workspace_for_ffn(T, W))
    mla.gated_ffn(x, W, outs[1], ws)
    mla.gated_ffn(x, W, outs[2], ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mla.gated_ffn(x, W, outs[3], ws, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(o, outs[0]) for o in outs[1:])


@pytest.mark.parametrize("four", [False, True], ids=["bf16w", "mx4"])
def test_graphs_that_share_a_workspace(four):
    """Two captured graphs and eager calls of other sizes on one workspace, replayed in turn."""
    mats = block(15, 512, 1376, four)
    W, L = mla.FfnWeights(*(m.device() for m in mats)), Matrix(16, 1000, 512, True).device()
    sizes = (7, 150)
    xs = [rows(17, T, 512).cuda() for T in sizes]
    ws = mla.workspace_for_ffn(300, W)
    lws = mla.workspace_for_linear4(300, L)
    big = torch.zeros(max(ws.numel(), lws.numel()), dtype=torch.uint8, device="cuda")
    outs = [(torch.empty((T, 512), dtype=F32, device="cuda"), torch.empty((T, 1000), dtype=BF16, device="cuda")) for T in sizes]

    def both(i):
        mla.gated_ffn(xs[i], W, outs[i][0], big)
        mla.linear4(xs[i], L, outs[i][1], big)

    both(0), both(1)
    torch.cuda.synchronize()
    want = [tuple(o.clone() for o in p) for p in outs]
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            both(i)
        graphs.append(g)
    x300 = rows(18, 300, 512).cuda()
    o300 = torch.empty((300, 512), dtype=F32, device="cuda")
    for turn in range(4):
        for i in (0, 1, 1, 0):
            for o in outs[i]:
                o.fill_(-1.0)
            graphs[i].replay()
            mla.gated_ffn(x300, W, o300, big)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i])), (turn, i)
        for x in xs:  # new inputs in place: a graph reads them as they are
            x.copy_(x.flip(0))
        both(0), both(1)
        torch.cuda.synchronize()
        want = [tuple(o.clone() for o in p) for p in outs]


@pytest.mark.parametrize("four", [False, True], ids=["bf16w", "mx4"])
def test_chunk_of_4160_rows(four):
    """The rows of 64 decodes and four 1024-token chunks, against 64-bit products of sampled rows."""
    log(f"[gpu] ffn 4160 rows {four}")
    T, hidden, inner = 4160, 2048, 1376
    x, mats = rows(19, T, hidden), block(20, hidden, inner, four)
    W = mla.FfnWeights(*(m.device() for m in mats))
    at = np.unique(np.concatenate(([0, 1, 255, 256, 4095, 4096, 4159], np.random.default_rng(0).integers(0, T, 60))))
    for dtype in (BF16, F32):
        out = torch.empty((T, hidden), dtype=dtype, device="cuda")
        mla.gated_ffn(x.cuda(), W, out, mla.workspace_for_ffn(T, W))
        ref = O.ffn(x[at].double().numpy(), *(m.values for m in mats), 3 if dtype == F32 else 1)
        assert_within(out[torch.from_numpy(at).cuda()].double().cpu().numpy(), *ref, dtype, f"{dtype}")


def test_offsets_beyond_32_bits():
    """An output of more than 2^32 bytes, the last rows and columns of it."""
    T, k, n = 66_000, 32, 33_000
    log("[gpu] linear4 66000 x 32 -> 33000")
    x, w = rows(21, T, k), Matrix(22, n, k, True)
    W = w.device()
    out = torch.empty((T, n), dtype=BF16, device="cuda")
    mla.linear4(x.cuda(), W, out, mla.workspace_for_linear4(T, W))
    at = np.array([0, 1, 32_537, 65_073, 65_074, T - 257, T - 1])
    ref = O.linear(x[at].double().numpy(), w.values)
    assert_within(out[torch.from_numpy(at).cuda()].double().cpu().numpy(), *ref, BF16, "sampled rows")


@pytest.mark.parametrize("T", [2, 40, 400])
def test_weights4_beyond_32_bits(T):
    """Codes of more than 2^32 bytes; the last output columns of them."""
    k, n = 131_072, 66_000
    log(f"[gpu] linear4 {T} x {k} -> {n}")
    gen = torch.Generator(device="cuda").manual_seed(51)
    W = mla.Weights4(torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda", generator=gen),
                     torch.randint(118, 122, (n, k // 32), dtype=torch.uint8, device="cuda", generator=gen))
    x = rows(52, T, k)
    out = torch.empty((T, n), dtype=F32, device="cuda")
    mla.linear4(x.cuda(), W, out, mla.workspace_for_linear4(T, W))
    cols, at = torch.tensor([0, 1, 32_767, 32_768, 65_537, n - 2, n - 1]), np.unique([0, T // 2, T - 1])
    values = O.mx4_values(W.codes[cols.cuda()].cpu().numpy(), W.scales[cols.cuda()].cpu().numpy())
    got = out[:, cols.cuda()].double().cpu().numpy()[at]
    assert_within(got, *O.linear(x[at].double().numpy(), values), F32, "sampled columns")


@pytest.mark.parametrize("T", [2, 40, 400])
def test_block_beyond_32_bits(T):
    """bf16 weights of more than 2^32 bytes each: of the inner width only the last 64 count, the other rows of gate and
    up are zero."""
    hidden, inner, last = 32_768, 66_000, 64
    log(f"[gpu] ffn {T} x {hidden} x {inner}")
    mats = block(53, hidden, last, False)
    gate, up = (torch.zeros((inner, hidden), dtype=BF16, device="cuda") for _ in range(2))
    gate[-last:], up[-last:] = mats[0].w.cuda(), mats[1].w.cuda()
    down = torch.ones((hidden, inner), dtype=BF16, device="cuda")
    down[:, -last:] = mats[2].w.cuda()
    W = mla.FfnWeights(gate, up, down)
    x = rows(54, T, hidden)
    out = torch.empty((T, hidden), dtype=F32, device="cuda")
    mla.gated_ffn(x.cuda(), W, out, mla.workspace_for_ffn(T, W))
    at = np.unique([0, T // 2, T - 1])
    assert_within(out.double().cpu().numpy()[at], *O.ffn(x[at].double().numpy(), *(m.values for m in mats), 3), F32, "sampled rows")


def test_rows_beyond_32_bits():
    """x of more than 2^32 bytes, and more rows than a launch counts in 16-row tiles along one of its axes."""
    T, k, n = 1_100_000, 2048, 32
    log(f"[gpu] linear4 {T} x {k} -> {n}")
    gen = torch.Generator(device="cuda").manual_seed(55)
    x = torch.randn((T, k), device="cuda", generator=gen, dtype=BF16)
    w = Matrix(56, n, k, True)
    W = w.device()
    out = torch.empty((T, n), dtype=F32, device="cuda")
    mla.linear4(x, W, out, mla.workspace_for_linear4(T, W))
    at = torch.tensor([0, 1, 1_048_575, 1_048_576, T - 2, T - 1], device="cuda")
    assert_within(out[at].double().cpu().numpy(), *O.linear(x[at].double().cpu().numpy(), w.values), F32, "sampled rows")


def test_rows_and_weights_at_other_alignments():
    """Views that start 16 bytes into a buffer; one that starts 2 bytes in is refused."""
    mats = block(23, 96, 160, False)
    x = rows(24, 9, 96)
    want = ffn(x, mats, F32)
    buf = torch.zeros(9 * 96 + 8, dtype=BF16, device="cuda")
    view = buf[8:].view(9, 96)
    view.copy_(x)
    gbuf = torch.zeros(160 * 96 + 8, dtype=BF16, device="cuda")
    gview = gbuf[8:].view(160, 96)
    gview.copy_(mats[0].w)
    W = mla.FfnWeights(gview, mats[1].device(), mats[2].device())
    out = torch.empty((9, 96), dtype=F32, device="cuda")
    mla.gated_ffn(view, W, out, mla.workspace_for_ffn(9, W))
    torch.cuda.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), want)
    odd = buf[1:1 + 9 * 96].view(9, 96)
    with pytest.raises(mla.MlaError):
        mla.gated_ffn(odd, W, out, mla.workspace_for_ffn(9, W))


def test_refusals_on_the_device():
    W = Matrix(25, 40, 64, True).device()
    x, out = rows(26, 5, 64).cuda(), torch.empty((5, 40), dtype=F32, device="cuda")
    ws = mla.workspace_for_linear4(5, W)
    for a in ((x.float(), W, out, ws), (x[:, :32], W, out, ws), (x[::2], W, out[::2], ws), (x, W, out[:4], ws), (x, W, out.half(), ws),
              (x.cpu(), W, out, ws), (x, W, out.cpu(), ws), (x, W, out, ws.cpu()), (x[0], W, out, ws), (x, W, out.T, ws)):
        with pytest.raises((ValueError, TypeError)):
            mla.linear4(*a)
    for short in (None, ws[:16], ws[:0]):
        with pytest.raises(mla.MlaError):
            mla.linear4(x, W, out, short)
    mla.linear4(x[:0], W, out[:0], None)


def test_an_attention_layer_and_its_feed_forward_half():
    """One step of a layer as a program runs it: attention layer, then the feed-forward block on its output, in
    bf16 and in 4 bits, against the oracle on the attention's own output."""
    from paper_2607_02043_amd import workloads as W_
    wl = W_.config(1)
    db = mla.DeviceBatch.from_batch(wl.batch)
    T = wl.batch.num_rows
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda()  # noqa: E731
    hidden, pool = up(W_.random_hidden(T, seed=0)), up(wl.layer(0).pool)
    mid = torch.empty((T, 2048), dtype=BF16, device="cuda")
    mla.mla_attention_layer(db, hidden, mla.DeviceProjWeights(W_.make_proj_weights(seed=0)), pool, W_.SOFTMAX_SCALE, mid,
                            mla.layer_workspace_for(db))
    for four in (False, True):
        mats = block(27, 2048, 1408, four)
        W = mla.FfnWeights(*(m.device() for m in mats))
        out = torch.empty((T, 2048), dtype=F32, device="cuda")
        mla.gated_ffn(mid, W, out, mla.workspace_for_ffn(T, W))
        torch.cuda.synchronize()
        ref = O.ffn(mid.double().cpu().numpy(), *(m.values for m in mats), 3)
        assert_within(out.double().cpu().numpy(), *ref, F32, f"four bits: {four}")
