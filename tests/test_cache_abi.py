"""The compact cache's entry points without a GPU: exported as declared, and
every bad argument refused on the host with a message."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2607_02043_amd as mla
from test_abi import FAKE, ROOT, _HostBatch

HEADER = os.path.join(ROOT, "include", "mla_cache.h")
INV, UNS = mla.MLA_ERR_INVALID_ARG, mla.MLA_ERR_UNSUPPORTED


def _err():
    return mla.lib().mla_last_error().decode()


def test_exports_and_constants():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"^(?:int|size_t)\s+(\w+)\s*\(", text, re.M))
    assert names == set(mla.EXPORTED_CACHE)
    for n in names:
        assert hasattr(mla.lib(), n)
    assert int(re.search(r"#define MLA_CACHE8_BLOCK (\d+)", text).group(1)) == mla.MLA_CACHE8_BLOCK


def cache(data=FAKE, scales=FAKE):
    return ctypes.byref(mla.mla_cache8(data=data, scales=scales))


def window(w, s):
    return ctypes.byref(mla.mla_window(w, s))


def append_rope(b, new=FAKE, base=10000.0, kv=FAKE):
    return mla.lib().append_latent_kv_rope(ctypes.byref(b.c), new, base, kv, None)


def append8(b, new=FAKE, base=10000.0, c=None):
    return mla.lib().append_latent_kv8(ctypes.byref(b.c), new, base, c if c is not None else cache(), None)


def attn8(b, q=FAKE, c=None, win=None, scale=0.07, out=FAKE, dtype=0, lse=None):
    return mla.lib().mixed_step_attn8(ctypes.byref(b.c), q, c if c is not None else cache(), win, scale, out, dtype, lse, None, 0, None)


def attnw(b, q=FAKE, kv=FAKE, win=None, scale=0.07, out=FAKE, dtype=0, lse=None):
    return mla.lib().mixed_step_attn_window(ctypes.byref(b.c), q, kv, win if win is not None else window(4, 0), scale, out, dtype, lse,
                                            None, 0, None)


ALL = (append_rope, append8, attn8, attnw)


@pytest.mark.parametrize("call", ALL)
def test_batches(call):
    assert call(_HostBatch([], [])) == mla.MLA_OK
    assert call(_HostBatch([0], [3])) == INV and "q_lens" in _err()
    assert call(_HostBatch([1], [-1])) == INV
    assert call(_HostBatch([5], [4092])) == INV and "exceeds" in _err()
    assert call(_HostBatch([1], [3], page=48)) == UNS
    b = _HostBatch([1], [3])
    b.c.block_table_dev = None
    assert call(b) == INV


def test_null_batch():
    L = mla.lib()
    assert L.append_latent_kv_rope(None, FAKE, 1e4, FAKE, None) == INV
    assert L.append_latent_kv8(None, FAKE, 1e4, cache(), None) == INV
    assert L.mixed_step_attn8(None, FAKE, cache(), None, 0.1, FAKE, 0, None, None, 0, None) == INV
    assert L.mixed_step_attn_window(None, FAKE, FAKE, window(1, 0), 0.1, FAKE, 0, None, None, 0, None) == INV
    assert L.mixed_step_attn8_workspace_bytes(None, None) == 0 and _err()


@pytest.mark.parametrize("base", [1.0, 0.5, -3.0, float("inf"), float("nan")])
def test_bad_base(base):
    b = _HostBatch([1], [3])
    assert append_rope(b, base=base) == INV and "rope_base" in _err()
    assert append8(b, base=base) == INV and "rope_base" in _err()


def test_rotating_append_needs_a_base():
    assert append_rope(_HostBatch([1], [3]), base=0.0) == INV


@pytest.mark.parametrize("call", (append8, attn8))
@pytest.mark.parametrize("page", [1, 8])
def test_8_bit_cache_needs_pages_of_16(call, page):
    assert call(_HostBatch([1], [3], page=page)) == UNS and "16" in _err()
    assert mla.lib().mixed_step_attn8_workspace_bytes(ctypes.byref(_HostBatch([1], [3], page=page).c), None) == 0 and "16" in _err()


@pytest.mark.parametrize("call", (append8, attn8))
def test_cache_pointers(call):
    b = _HostBatch([1], [3])
    for bad in (cache(data=None), cache(scales=None), cache(data=FAKE + 8), cache(scales=FAKE + 4)):
        assert call(b, c=bad) == INV and "cache" in _err()
    assert mla.lib().append_latent_kv8(ctypes.byref(b.c), FAKE, 1e4, None, None) == INV


def test_other_pointers():
    b = _HostBatch([1], [3])
    for kw in (dict(new=None), dict(new=FAKE + 2), dict(kv=None), dict(kv=FAKE + 8)):
        assert append_rope(b, **kw) == INV, kw
    for kw in (dict(new=None), dict(new=FAKE + 8)):
        assert append8(b, **kw) == INV, kw
    for kw in (dict(q=None), dict(q=FAKE + 2), dict(out=None), dict(out=FAKE + 4), dict(lse=FAKE + 2), dict(dtype=2), dict(dtype=-1),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attn8(b, **kw) == INV, kw
        assert attnw(b, **kw) == INV, kw
    assert attnw(b, kv=None) == INV and attnw(b, kv=FAKE + 8) == INV


@pytest.mark.parametrize("w,s", [(0, 0), (-1, 4), (5, -1)])
def test_bad_windows(w, s):
    b = _HostBatch([1], [3])
    assert attn8(b, win=window(w, s)) == INV
    assert attnw(b, win=window(w, s)) == INV
    for f in (mla.lib().mixed_step_attn8_workspace_bytes, mla.lib().mixed_step_attn_window_workspace_bytes):
        assert f(ctypes.byref(b.c), window(w, s)) == 0 and _err()
    assert mla.lib().mixed_step_attn_window(ctypes.byref(b.c), FAKE, FAKE, None, 0.07, FAKE, 0, None, None, 0, None) == INV
    assert mla.lib().mixed_step_attn_window_workspace_bytes(ctypes.byref(b.c), None) == 0 and "NULL" in _err()


def test_scale_bytes():
    f = mla.lib().mla_cache8_scale_bytes
    assert [f(1, 16), f(5, 16), f(4, 16), f(3, 64), f(1, 1024)] == [16, 32, 16, 48, 256]
    assert [f(0, 64), f(-1, 64), f(4, 8), f(4, 48), f(4, 2048)] == [0] * 5


def test_python_cache_and_its_refusals():
    c = mla.LatentCache8(num_pages=3, page_size=32, device="cpu")
    assert c.data.shape == (3, 32, 576) and c.scales.shape == (3, 2, 2) and c.scales.dtype == torch.bfloat16
    assert (c.data == 0).all() and (c.scales == 1).all()
    assert c.scales.untyped_storage().nbytes() == 32
    for n, P in ((0, 64), (4, 8), (4, 48)):
        with pytest.raises(ValueError):
            mla.LatentCache8(num_pages=n, page_size=P, device="cpu")
    d, s = torch.zeros((3, 32, 576), dtype=torch.uint8), torch.ones((3, 2, 2), dtype=torch.bfloat16)
    assert mla.LatentCache8(data=d, scales=s).num_pages == 3
    for dd, ss in ((d[:, :, :512], s), (d.to(torch.int16), s), (d, s[:2]), (d, s.float()), (d[:, ::2], s[:, :1]), (d, s.transpose(0, 1))):
        with pytest.raises(ValueError):
            mla.LatentCache8(data=dd, scales=ss)
    b = mla.DeviceBatch([1], [3], np.zeros((1, 1)), 64, 3, device="cpu")
    with pytest.raises(ValueError):  # pages of another size
        mla.append_latent_kv8(b, torch.zeros((1, 576), dtype=torch.bfloat16), c)
    b = mla.DeviceBatch([1], [3], np.zeros((1, 1)), 32, 4, device="cpu")
    with pytest.raises(ValueError):  # fewer pages than the batch's pool
        mla.append_latent_kv8(b, torch.zeros((1, 576), dtype=torch.bfloat16), c)


def test_python_refuses_other_shapes_and_strides():
    b = mla.DeviceBatch([1, 2], [3, 0], np.zeros((2, 1)), 32, 3, device="cpu")
    c = mla.LatentCache8(num_pages=3, page_size=32, device="cpu")
    bf = dict(dtype=torch.bfloat16)
    new, kv = torch.zeros((3, 576), **bf), torch.zeros((3, 32, 576), **bf)
    q, out = torch.zeros((3, 16, 576), **bf), torch.zeros((3, 16, 512))
    for bad in (new[:2], torch.zeros((3, 1152), **bf)[:, ::2], new.float()):
        with pytest.raises(ValueError):
            mla.append_latent_kv_rope(b, bad, 1e4, kv)
        with pytest.raises(ValueError):
            mla.append_latent_kv8(b, bad, c)
    for bad in (kv[:2], kv[:, :16], kv.float(), kv.transpose(0, 1).contiguous().transpose(0, 1)):
        with pytest.raises(ValueError):
            mla.append_latent_kv_rope(b, new, 1e4, bad)
        with pytest.raises(ValueError):
            mla.mixed_step_attn_window(b, q, bad, (4, 0), 0.07, out)
    for kw in (dict(q=q[:2]), dict(q=q.float()), dict(out=out[:, :, :256]), dict(out=out.double()), dict(lse=torch.zeros(3, 8)),
               dict(q=torch.zeros((16, 3, 576), **bf).transpose(0, 1))):
        a = dict(dict(q=q, out=out, lse=None), **kw)
        with pytest.raises((ValueError, TypeError)):
            mla.mixed_step_attn8(b, a["q"], c, 0.07, a["out"], a["lse"])
        with pytest.raises((ValueError, TypeError)):
            mla.mixed_step_attn_window(b, a["q"], kv, (4, 0), 0.07, a["out"], a["lse"])


def test_python_refuses_other_types_devices_and_windows():
    b = mla.DeviceBatch([1, 2], [3, 0], np.zeros((2, 1)), 32, 3, device="cpu")
    c = mla.LatentCache8(num_pages=3, page_size=32, device="cpu")
    new, q, out = torch.zeros((3, 576), dtype=torch.bfloat16), torch.zeros((3, 16, 576), dtype=torch.bfloat16), torch.zeros((3, 16, 512))
    with pytest.raises(ValueError, match="batch is on cpu"):
        mla.append_latent_kv8(b, new, c)
    with pytest.raises(ValueError, match="float16"):
        mla._dev(new.half(), "new_latents", (3, 576), mla._bf16(), 0)
    with pytest.raises(ValueError, match="on cpu"):
        mla._dev(new, "new_latents", (3, 576), mla._bf16(), 0)
    for data, scales in ((c.data.bool(), c.scales), (c.data.view(torch.int8), c.scales), (c.data, c.scales.half())):
        with pytest.raises(ValueError):
            mla.LatentCache8(data=data, scales=scales)
    for w in ((1 << 31, 0), ((1 << 32) + 5, 0), (4, 1 << 32), (-(1 << 40), 0)):
        with pytest.raises(ValueError, match="32 bits"):
            mla.workspace_for_cache8(b, window=w)
        with pytest.raises(ValueError, match="32 bits"):
            mla.workspace_for_window(b, w)
