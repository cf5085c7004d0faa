"""An attention layer on the compact latent cache, as a program writes it: projections, append,
attention, output projection (needs an MI355X).  Each stage is checked on what the stage before
it left on the GPU; a captured layer replays the same bits."""
import numpy as np
import pytest

import cache_cases as C
import paper_2607_02043_amd as mla
from harness import from_dev_u16, log, to_dev
from oracle import cache_oracle as CO
from oracle import proj_oracle as PO
from paper_2607_02043_amd import workloads as W
from test_gpu_cache import SCALE, Attend, dev_cache, down8, flags  # noqa: F401  (flags: a fixture)
from test_gpu_layer import _gemm_bound, weights  # noqa: F401  (weights: a fixture)

pytestmark = pytest.mark.gpu


class Layer:
    """The buffers of one step and the four calls on them."""

    def __init__(self, b, hidden, dw, cache, window, bf16):
        import torch
        T = b.num_rows
        self.a = Attend(b, np.zeros((T, 16, 576), np.uint16), *down8(cache), window=window, bf16=bf16)
        self.a.cache = cache
        self.dw, self.cache, self.window = dw, cache, window
        self.hidden, self.new = to_dev(hidden), torch.empty((T, 576), dtype=torch.int16, device="cuda")
        self.out = torch.empty((T, 2048), dtype=torch.float32, device="cuda")
        self.proj = torch.empty(mla.mla_proj_workspace_bytes(T), dtype=torch.uint8, device="cuda")

    def run(self):
        a = self.a
        mla.mla_pre_attn(a.db, self.hidden, self.dw, a.qd, self.new, self.proj)
        mla.append_latent_kv8(a.db, self.new, self.cache)  # (pre_attn has rotated them)
        mla.mixed_step_attn8(a.db, a.qd, self.cache, SCALE, a.out, a.lse, a.ws, window=self.window)
        mla.mla_post_attn(a.out, self.dw, self.out, self.proj)


@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("window", [None, (48, 4)], ids=str)
def test_layers_on_the_8_bit_cache(window, bf16, weights):  # noqa: F811
    import torch
    _, wo, dw = weights
    P, n_req = 16, 3
    table = np.random.default_rng(5).permutation(48).astype(np.int32).reshape(n_req, 16)
    lens = np.array([0, 61, 130])
    cache = dev_cache(*C.cache8(W.Batch(P, lens.astype(np.int32), np.ones(n_req, np.int32), table, 48), 6))
    for step, rows in enumerate([[35, 1, 1], [18, 1, 2], [1, 1, 1]]):
        b = W.Batch(P, lens.astype(np.int32), np.array(rows, np.int32), table, 48)
        hidden = W.random_hidden(b.num_rows, seed=50 + step)
        log(f"[gpu] layer step {step}: rows {rows}, window {window}, bf16 {bf16}")
        before = down8(cache)
        s = Layer(b, hidden, dw, cache, window, bf16)
        s.run()
        torch.cuda.synchronize()
        # projections, against the oracle's stored values: a flip is one step of bf16
        q_ref, lat_ref = PO.pre_attn(PO.positions(b.q_lens, b.prefix_lens), PO.bf16_value(hidden), wo, rounded=True)
        q, lat = from_dev_u16(s.a.qd), from_dev_u16(s.new)
        assert (q != q_ref).mean() <= 0.01 and (lat != lat_ref).mean() <= 0.01
        # the append, bit for bit
        want, ws, _ = CO.append8(b, lat, 0.0, *before)
        data, scales = down8(cache)
        np.testing.assert_array_equal(scales.reshape(-1, 2), ws)
        np.testing.assert_array_equal(data.reshape(-1, 576), want)
        # the attention over what the cache holds now
        s.a.q, s.a.data, s.a.scales = q, data, scales
        s.a.keys = lambda r, n: CO.keys8(b, r, n, data, scales)
        s.a.check(f"attention of step {step}")
        # the output projection: o rounds to bf16 once, the sums are fp32
        ab = PO.through_bf16(s.a.results()[0])
        o = np.concatenate([ab[:, h] @ wo.w_uv[h].T for h in range(16)], axis=1)
        up, mags = _gemm_bound(o, wo.w_o)
        assert (np.abs(s.out.double().cpu().numpy() - o @ wo.w_o.T) <= up + 2.0 ** -16 * mags).all()
        # captured: the append finds its own tokens and leaves the same bytes
        first = [x.clone() for x in (s.out, s.a.lse, cache.data, cache.scales)]
        g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(g, stream=side):
            s.run()
        for _ in range(3):
            s.out.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip(first, (s.out, s.a.lse, cache.data, cache.scales)):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
            s.run()
        lens = lens + np.array(rows)
    assert mla.device_flags() == 0


def test_layer_through_a_window_of_the_bf16_cache(weights):  # noqa: F811
    """pre_attn's latents are rotated: append_latent_kv, then attention through the window."""
    import torch
    _, wo, dw = weights
    window = (40, 3)
    b = C.batch([100, 0, 77], [1, 50, 1], 32, seed=51)
    rng = np.random.default_rng(51)
    pool = W.f32_to_bf16_bits(rng.standard_normal((b.num_pages, 32, 576), dtype=np.float32))
    hidden = W.random_hidden(b.num_rows, seed=52)
    a = Attend(b, np.zeros((b.num_rows, 16, 576), np.uint16), pool=pool, window=window)
    new = torch.empty((b.num_rows, 576), dtype=torch.int16, device="cuda")
    ws = torch.empty(mla.mla_proj_workspace_bytes(b.num_rows), dtype=torch.uint8, device="cuda")
    out = torch.empty((b.num_rows, 2048), dtype=torch.float32, device="cuda")
    mla.mla_pre_attn(a.db, to_dev(hidden), dw, a.qd, new, ws)
    mla.append_latent_kv(a.db, new, a.cache)
    a.run()
    mla.mla_post_attn(a.out, dw, out, ws)
    a.q, after = from_dev_u16(a.qd), from_dev_u16(a.cache)
    a.keys = lambda r, n: CO.keys16(b, r, n, after)
    a.check("attention")
    ab = PO.through_bf16(a.results()[0])
    o = np.concatenate([ab[:, h] @ wo.w_uv[h].T for h in range(16)], axis=1)
    up, mags = _gemm_bound(o, wo.w_o)
    assert (np.abs(out.double().cpu().numpy() - o @ wo.w_o.T) <= up + 2.0 ** -16 * mags).all()
    assert mla.device_flags() == 0
