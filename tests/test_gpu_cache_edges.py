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
