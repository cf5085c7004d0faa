"""The feed-forward entry points without a GPU: exported as declared, and every bad
argument refused on the host with a message."""
import ctypes
import os
import re

import pytest
import torch

import paper_2607_02043_amd as mla
from test_abi import FAKE, ROOT

HEADER = os.path.join(ROOT, "include", "mla_ffn.h")
INV, UNS, WS = mla.MLA_ERR_INVALID_ARG, mla.MLA_ERR_UNSUPPORTED, mla.MLA_ERR_WORKSPACE
BIG = 1 << 45


def _err():
    return mla.lib().mla_last_error().decode()


def test_exports_and_constants():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"^(?:int|size_t)\s+(\w+)\s*\(", text, re.M))
    assert names == set(mla.EXPORTED_FFN)
    for n in names:
        assert hasattr(mla.lib(), n)
    for name in ("MLA_MX4_GROUP", "MLA_FFN_COUNTER_BYTES"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(mla, name)


def mx4(codes=FAKE, scales=FAKE):
    return mla.mla_mx4(codes, scales)


def linear(T=3, x=FAKE, w=None, k=64, n=24, out=FAKE, dtype=0, ws=FAKE, ws_bytes=BIG, null_w=False):
    p = None if null_w else ctypes.byref(w if w is not None else mx4())
    return mla.lib().mla_linear4(T, x, p, k, n, out, dtype, ws, ws_bytes, None)


def ffn(T=3, x=FAKE, w=None, k=64, n=32, out=FAKE, dtype=0, ws=FAKE, ws_bytes=BIG, null_w=False, ptrs=(FAKE, FAKE, FAKE)):
    p = None if null_w else ctypes.byref(mla.mla_ffn_weights(*ptrs, k, n))
    return mla.lib().mla_gated_ffn(T, x, p, out, dtype, ws, ws_bytes, None)


def ffn4(T=3, x=FAKE, w=None, k=64, n=32, out=FAKE, dtype=0, ws=FAKE, ws_bytes=BIG, null_w=False, ptrs=None):
    p = None if null_w else ctypes.byref(mla.mla_ffn4_weights(*(ptrs or (mx4(), mx4(), mx4())), k, n))
    return mla.lib().mla_gated_ffn4(T, x, p, out, dtype, ws, ws_bytes, None)


ALL = (linear, ffn, ffn4)


@pytest.mark.parametrize("call", ALL)
def test_arguments(call):
    assert call(T=0, x=None, out=None, ws=None) == mla.MLA_OK and _err() == ""
    assert call(T=-1) == INV and "num_rows" in _err()
    for bad in (None, FAKE + 8):
        assert call(x=bad) == INV and "x / out" in _err()
        assert call(out=bad) == INV and "x / out" in _err()
        assert call(ws=bad) == WS and "workspace" in _err()
    for dtype in (-1, 2):
        assert call(dtype=dtype) == INV and "out_dtype" in _err()
    assert call(null_w=True) == INV and _err()
    for size in ("k", "n"):
        for v in (0, -8):
            assert call(**{size: v}) == INV and "< 1" in _err()
        for v in (4, 33, 12, (1 << 24) + 32):
            assert call(**{size: v}) == UNS and "multiple" in _err()


def test_weights():
    for bad in (None, FAKE + 1):
        assert linear(w=mx4(codes=bad)) == INV and "codes and scales of w" in _err()
        assert linear(w=mx4(scales=bad)) == INV
        for i, name in enumerate(("w_gate", "w_up", "w_down")):
            ptrs = [FAKE] * 3
            ptrs[i] = bad
            assert ffn(ptrs=ptrs) == INV and name in _err()
            four = [mx4(), mx4(), mx4()]
            four[i] = mx4(scales=bad)
            assert ffn4(ptrs=four) == INV and name in _err()
    assert ffn4(k=40) == UNS and ffn4(n=40) == UNS and linear(k=40) == UNS


def test_workspace_sizes():
    L = mla.lib()
    for T, k, n in ((1, 64, 32), (33, 2048, 1408), (4160, 2048, 10944), (70000, 256, 32)):
        need = L.mla_gated_ffn_workspace_bytes(T, k, n)
        assert need >= mla.MLA_FFN_COUNTER_BYTES + T * n * 6
        assert ffn(T=T, k=k, n=n, ws_bytes=need - 1) == WS and str(need) in _err()
        assert ffn4(T=T, k=k, n=n, ws_bytes=need - 1) == WS
        need = L.mla_linear4_workspace_bytes(T, k, n)
        assert need >= mla.MLA_FFN_COUNTER_BYTES
        assert linear(T=T, k=k, n=n, ws_bytes=need - 1) == WS
    for f in (L.mla_gated_ffn_workspace_bytes, L.mla_linear4_workspace_bytes):
        assert f(0, 64, 32) == 0 and f(-1, 64, 32) == 0 and f(3, 60, 32) == 0 and f(3, 64, 12) == 0 and f(3, 0, 32) == 0
        sizes = [f(T, 2048, 1408) for T in range(1, 700)] + [f(T, 2048, 1408) for T in (1000, 2000, 5000, 20000)]
        assert sizes == sorted(sizes), "a workspace for more rows serves fewer"


def _w4(n, k):
    return mla.Weights4(torch.zeros((n, k // 2), dtype=torch.uint8), torch.zeros((n, k // 32), dtype=torch.uint8))


def test_weights4_refuses():
    codes, scales = torch.zeros((8, 32), dtype=torch.uint8), torch.zeros((8, 2), dtype=torch.uint8)
    w = mla.Weights4(codes, scales)
    assert (w.out_features, w.in_features) == (8, 64) and w.c.codes == codes.data_ptr() and w.c.scales == scales.data_ptr()
    for c, s in ((codes.to(torch.int8), scales), (codes[:, :24], scales), (codes[:, :0], scales[:, :0]), (codes.T, scales),
                 (codes[None], scales), (codes, scales[:, :1]), (codes, scales.to(torch.int8)), (codes, scales.T.contiguous()),
                 (codes[::2], scales[::2])):
        with pytest.raises(ValueError):
            mla.Weights4(c, s)
    with pytest.raises(AttributeError):
        w.codes = codes


def test_ffn_weights_refuse():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    w = mla.FfnWeights(bf(40, 24), bf(40, 24), bf(24, 40))
    assert (w.hidden, w.inner, w.four_bit) == (24, 40, False)
    w = mla.FfnWeights(_w4(32, 64), _w4(32, 64), _w4(64, 32))
    assert (w.hidden, w.inner, w.four_bit) == (64, 32, True)
    for g, u, d in ((bf(40, 24), bf(40, 24), bf(40, 24)), (bf(40, 24), bf(32, 24), bf(24, 40)), (bf(40, 24).float(), bf(40, 24), bf(24, 40)),
                    (bf(24, 40).T, bf(40, 24), bf(24, 40)), (bf(40, 24), bf(40, 24).half(), bf(24, 40)), (bf(960), bf(960), bf(960)),
                    (_w4(32, 64), bf(32, 64), bf(64, 32)), (bf(32, 64), bf(32, 64), _w4(64, 32)), (_w4(32, 64), _w4(32, 64), _w4(32, 64))):
        with pytest.raises(ValueError):
            mla.FfnWeights(g, u, d)
    with pytest.raises(AttributeError):
        w.gate = w.up


def test_tensors_that_are_not_on_the_device():
    with pytest.raises(ValueError):
        mla.linear4(torch.zeros((2, 64), dtype=torch.bfloat16), _w4(8, 64), torch.zeros((2, 8)), None)
    with pytest.raises(ValueError):
        mla.workspace_for_linear4(3, _w4(12, 64), device="cpu")
    assert mla.workspace_for_linear4(0, _w4(8, 64), device="cpu") is None
    ws = mla.workspace_for_ffn(5, mla.FfnWeights(_w4(32, 64), _w4(32, 64), _w4(64, 32)), device="cpu")
    assert ws.numel() == mla.lib().mla_gated_ffn_workspace_bytes(5, 64, 32) and not ws[:mla.MLA_FFN_COUNTER_BYTES].any()
