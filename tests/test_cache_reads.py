"""What the attention over the 8-bit cache reads of the scales (host code, no GPU):
the four bytes of a block and nothing beside them, since the array of a program's own
pool may end right behind its last block."""
import os
import re

from paper_2607_02043_amd import build

HEADERS = ("cache_tile.h", "cache_decode.h", "cache_append.h")


def test_scales_are_read_four_bytes_at_a_time():
    text = {h: open(os.path.join(build.CSRC, h)).read() for h in HEADERS}
    text["mla_kernels.hip"] = open(os.path.join(build.CSRC, "mla_kernels.hip")).read()
    # their address is formed in one place, without rounding it down, and goes to the four-byte load alone
    uses = [(h, line.strip()) for h, t in text.items() for line in t.splitlines() if "kv8_scales" in line]
    assert uses == [("cache_tile.h", "return reinterpret_cast<const char *>(a.kv8_scales) + pool_slot / kBlock8 * 4;")], uses
    body = re.search(r"void dma_scales8\(.*?\n}", text["cache_tile.h"], re.S).group(0)
    assert "lds_dma4(" in body and "lds_dma16" not in body
    body = re.search(r"void lds_dma4\(.*?\n}", text["cache_tile.h"], re.S).group(0)
    assert "global_load_lds_dword %1" in body
    for h in ("cache_decode.h", "mla_kernels.hip"):
        calls = re.findall(r"(\w+)\([^;]*(?:block_scales8\(|s\.scale,)", text[h])
        assert calls and set(calls) <= {"dma_scales8"}, (h, calls)
