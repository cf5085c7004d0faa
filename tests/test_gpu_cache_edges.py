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
