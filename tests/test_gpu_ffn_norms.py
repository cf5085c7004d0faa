"""fp32 results of the feed-forward operators in the 2-norm (needs an MI355X): a third of h's bits, parts of
a split sum or outputs that were held in too few bits would show, as they do not within the bound
of each value for itself."""
import numpy as np
import pytest

from ffn_cases import Matrix, block, ffn, linear4, rows
from harness import log
from oracle import ffn_oracle as O
from test_gpu_ffn import EVERY_KERNEL, F32, FEW, LINEAR_SIZES, SIZES, SIZES4

pytestmark = pytest.mark.gpu


def _sample(T):
    edge = np.arange(0, T, 128)
    return np.unique(np.concatenate((np.arange(min(T, 8)), np.arange(max(0, T - 8), T), edge, edge[1:] - 1, np.random.default_rng(2).integers(0, T, 64))))


def _check(got, out, limit):
    rel = np.linalg.norm(got - out) / np.linalg.norm(out)
    log(f"[gpu] {rel:.2e} of {limit:.2e}")
    assert rel <= limit, f"off by {rel:.3g} in the 2-norm, at most {limit:.3g}"


PRODUCTS = [(T, k, n) for T in FEW for k, n in LINEAR_SIZES] + [(T, k, n) for what, T, k, n, f32 in EVERY_KERNEL if what == 0 and f32]
BLOCKS = [(four, T, k, n) for T in FEW for four, sizes in ((False, SIZES), (True, SIZES4)) for k, n in sizes]
BLOCKS += [(what == 2, T, k, n) for what, T, k, n, f32 in EVERY_KERNEL if what != 0 and f32]


@pytest.mark.parametrize("T,k,n", PRODUCTS)
def test_product(T, k, n):
    log(f"[gpu] product {T} x {k} -> {n}")
    x, w, at = rows(81, T, k), Matrix(82, n, k, True), _sample(T)
    _check(linear4(x, w, F32)[at], O.linear(x[at].double().numpy(), w.values)[0], O.linear_norm(k))


@pytest.mark.parametrize("four,T,hidden,inner", BLOCKS)
def test_block(four, T, hidden, inner):
    log(f"[gpu] block {T} x {hidden} x {inner} {four}")
    x, mats, at = rows(83, T, hidden), block(84, hidden, inner, four), _sample(T)
    _check(ffn(x, mats, F32)[at], O.ffn(x[at].double().numpy(), *(m.values for m in mats), 3)[0], O.ffn_norm(hidden, inner))
