"""Attention of the compact latent cache with bf16 output on the GPU: the tests of
fp32 output (test_gpu_cache.py, test_gpu_cache_edges.py), whose chunk rows run on kernels of
their own, with the other output type and its bounds."""
import pytest

import test_gpu_cache as T
import test_gpu_cache_edges as E
from test_gpu_cache import Attend, flags  # noqa: F401  (flags: a fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def bf16_output(monkeypatch):
    for m in (T, E):
        monkeypatch.setattr(m, "Attend", lambda *a, **k: Attend(*a, **{**k, "bf16": True}))


FORMS = [(True, None)] + [(e, w) for e in (True, False) for w in T.WINDOWS if w is not None]


@pytest.mark.parametrize("eight,window", FORMS, ids=str)
@pytest.mark.parametrize("name", T.BATCHES)
def test_attention(name, eight, window):
    T.test_attention(name, window, eight)


@pytest.mark.parametrize("page", [1, 2, 8])
@pytest.mark.parametrize("window", [(1, 0), (9, 3), (40, 33)], ids=str)
def test_window_on_small_pages(page, window):
    T.test_window_on_small_pages(page, window)


@pytest.mark.parametrize("case,eight", [(c, e) for c in T.LARGE for e in (True, False) if e or c[3] is not None], ids=T.ids)
def test_split_rows(case, eight):
    T.test_split_rows(*case, eight)


@pytest.mark.parametrize("eight", [True, False], ids=["8-bit", "bf16"])
def test_where_no_row_looks(eight):
    for page in (16, 64):
        T.test_nan_and_bad_pages_where_no_row_looks(eight, page)


@pytest.mark.parametrize("eight", [True, False], ids=["8-bit", "bf16"])
def test_a_nan_key_reaches_the_rows_that_see_it_alone(eight):
    T.test_a_nan_key_reaches_the_rows_that_see_it_alone(eight)


def test_scores_far_above_the_first_tiles():
    T.test_scores_far_above_the_first_tiles()


@pytest.mark.parametrize("window", [None, (130, 21)], ids=str)
@pytest.mark.parametrize("case", T.FAR, ids=T.ids)
@pytest.mark.parametrize("order", ["rising", "falling", "random"])
def test_scales_far_apart(order, case, window):
    T.test_scales_far_apart(*case, window, order)


@pytest.mark.parametrize("bits", [0x7FC0, 0xFF80, 0x0000])
@pytest.mark.parametrize("page", [16, 64])
def test_any_scale_where_no_row_looks(bits, page):
    T.test_any_scale_where_no_row_looks(bits, page)


@pytest.mark.parametrize("spread", [0.0, 1.0])
@pytest.mark.parametrize("prefix,rows,keys,unit", [([2500, 90], [1, 1], 0, 3), ([300], [20], 64, 0), ([1500, 0], [9, 33], 128, 0)], ids=str)
def test_split_rows_of_the_largest_values(prefix, rows, keys, unit, spread):
    E.test_split_rows_of_the_largest_values(prefix, rows, keys, unit, spread)


@pytest.mark.parametrize("keys,unit", [(0, 0), (64, 1)], ids=["whole", "split"])
@pytest.mark.parametrize("window", [(16, 2), (70, 3), (1 << 20, 0)], ids=str)
def test_infinities_of_a_windowed_cache(window, keys, unit):
    E.test_infinities_of_a_windowed_cache(window, keys, unit)
