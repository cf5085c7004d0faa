"""The bounds in the 2-norm on fp32 results (CPU): fp32 arithmetic keeps them, and a result whose
sums, h or output were held in fewer bits does not."""
import math

import numpy as np
import pytest
import torch

from oracle import ffn_oracle as O

SIZES = [(128, 160), (288, 416), (2048, 1408), (2048, 5504)]


def _rand(seed, *shape):
    return torch.from_numpy(np.random.default_rng([seed, *shape]).standard_normal(shape) / math.sqrt(shape[1])).to(torch.bfloat16)


def _two_planes(h):
    """h cut to its 16 leading bits."""
    return (h.view(torch.int32) & ~0xFF).view(torch.float32)


def _off(y, out):
    return float(np.linalg.norm(y.double().numpy() - out) / np.linalg.norm(out))


@pytest.mark.parametrize("hidden,inner", SIZES)
def test_block(hidden, inner):
    x, gate, up, down = _rand(1, 24, hidden) * math.sqrt(hidden), _rand(2, inner, hidden), _rand(3, inner, hidden), _rand(4, hidden, inner)
    out, _ = O.ffn(*(t.double().numpy() for t in (x, gate, up, down)), 3)
    g, u = x.float() @ gate.float().T, x.float() @ up.float().T
    h = g / (1 + torch.exp(-g)) * u
    y, limit = h @ down.float().T, O.ffn_norm(hidden, inner)
    assert _off(y, out) <= limit
    assert _off(_two_planes(h) @ down.float().T, out) > limit, "h of 16 bits"
    assert _off(h.to(torch.bfloat16).float() @ down.float().T, out) > limit, "h of 8 bits"
    assert _off(y.half(), out) > limit and _off(y.to(torch.bfloat16), out) > limit, "a rounded result"


@pytest.mark.parametrize("k", [32, 352, 2048, 10944])
def test_product(k):
    x, w = _rand(5, 40, k), _rand(6, 200, k)
    out, _ = O.linear(x.double().numpy(), w.double().numpy())
    y, limit = x.float() @ w.float().T, O.linear_norm(k)
    assert _off(y, out) <= limit
    assert _off(y.half(), out) > limit and _off(y.to(torch.bfloat16), out) > limit, "a rounded result"
    if k >= 352:  # four parts of K, each rounded
        edges = [k * i // 4 for i in range(5)]
        parts = [x.float()[:, a:b] @ w.float()[:, a:b].T for a, b in zip(edges, edges[1:])]
        assert _off(sum(p.half().float() for p in parts), out) > limit, "rounded parts"
