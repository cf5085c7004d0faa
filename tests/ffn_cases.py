"""Inputs and runs of the feed-forward operators for their tests."""
import math

import numpy as np
import torch

import paper_2607_02043_amd as mla
from oracle import ffn_oracle as O

GUARD = 3  # rows on either side of the output that a call leaves as they are


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.bfloat16)


def rows(seed, T, k):
    rng = np.random.default_rng([seed, T, k])
    return bf16(rng.standard_normal((T, k)) * np.exp(0.3 * rng.standard_normal(k)))


class Matrix:
    """A weight matrix [n][k], and its values in 64 bits."""

    def __init__(self, seed, n, k, four):
        w = np.random.default_rng([seed, n, k, 5]).standard_normal((n, k)) / math.sqrt(k)
        if four:
            codes, scales = O.mx4_quantize(w)
            self.codes, self.scales = torch.from_numpy(codes), torch.from_numpy(scales)
        else:
            self.w = bf16(w)
        self.four = four

    @property
    def values(self):
        return O.mx4_values(self.codes.numpy(), self.scales.numpy()) if self.four else self.w.double().numpy()

    def device(self):
        return mla.Weights4(self.codes.cuda(), self.scales.cuda()) if self.four else self.w.cuda()


def guarded(T, n, dtype):
    """(whole tensor filled with a pattern, the rows in its middle that a call writes)"""
    whole = torch.full((T + 2 * GUARD, n), 77.0, dtype=dtype, device="cuda")
    return whole, whole[GUARD:GUARD + T]


def finish(whole, T, ws):
    """The result in 64 bits, after the checks that nothing else changed."""
    torch.cuda.synchronize()
    assert bool((whole[:GUARD] == 77).all()) and bool((whole[GUARD + T:] == 77).all()), "rows beside the output changed"
    assert not bool(ws[:mla.MLA_FFN_COUNTER_BYTES].any()), "counters are not zero after the call"
    return whole[GUARD:GUARD + T].double().cpu().numpy()


def fenced(ws):
    """The workspace inside a larger buffer of ones, so that writes behind it show."""
    big = torch.full((ws.numel() + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    big[:mla.MLA_FFN_COUNTER_BYTES] = 0
    return big, big[:ws.numel()]


def linear4(x, w, dtype):
    T = x.shape[0]
    W = w.device()
    whole, out = guarded(T, W.out_features, dtype)
    big, ws = fenced(mla.workspace_for_linear4(T, W))
    mla.linear4(x.cuda(), W, out, ws)
    got = finish(whole, T, ws)
    assert bool((big[ws.numel():] == 0xFF).all()), "written behind the workspace"
    return got


def ffn(x, mats, dtype):
    T = x.shape[0]
    W = mla.FfnWeights(*(m.device() for m in mats))
    whole, out = guarded(T, W.hidden, dtype)
    big, ws = fenced(mla.workspace_for_ffn(T, W))
    mla.gated_ffn(x.cuda(), W, out, ws)
    got = finish(whole, T, ws)
    assert bool((big[ws.numel():] == 0xFF).all()), "written behind the workspace"
    return got


def block(seed, hidden, inner, four):
    return Matrix(seed, inner, hidden, four), Matrix(seed + 1, inner, hidden, four), Matrix(seed + 2, hidden, inner, four)


def assert_within(got, ref, bound, dtype, what):
    tol = O.rounded_bound(ref, bound, dtype == torch.bfloat16)
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN elsewhere"
    assert np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)]), f"{what}: infinities"
    off = np.abs(got - ref)[fine] / np.maximum(tol[fine], 1e-300)
    worst = float(off.max()) if off.size else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} of the bound, {int((off > 1).sum())} of {off.size} values"
