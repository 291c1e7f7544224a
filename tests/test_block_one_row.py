"""Calls of one token row: their row strides are not looked at (include/moev.h).  No GPU: no sequence, so nothing is launched."""
import ctypes as C

import pytest

import paper_2607_12696_b200 as moev
from test_block_args import BASE, batch, cache

L = moev.lib()


@pytest.mark.parametrize("stride", [0, 3, 5, -7, 129])
@pytest.mark.parametrize("rows", [0, 1])
def test_strides_of_one_row_are_not_looked_at(stride, rows):
    c, b = C.byref(cache()), C.byref(batch(n_seq=0, n_tokens=rows))
    assert L.moev_cache_append(c, b, BASE, stride, BASE, stride, None, 0, BASE, stride, 4, BASE, stride, None) == 0
    assert L.moev_cache_attend(c, b, BASE, stride, 4, 0.1, 0, None, BASE, stride, None, BASE, 1 << 40, None) == 0


@pytest.mark.parametrize("stride", [0, 3, 120, 257])
def test_strides_of_more_rows_are(stride):
    c, b = C.byref(cache()), C.byref(batch(n_seq=0, n_tokens=2))
    ok = dict(k=128, v=128, q=256, o=256)
    for name in ok:
        s = {**ok, name: stride}
        assert L.moev_cache_append(c, b, BASE, s["k"], BASE, s["v"], None, 0, BASE, s["q"], 4, BASE, s["o"], None) == 1
    for q, o in ((stride, 256), (256, stride)):
        assert L.moev_cache_attend(c, b, BASE, q, 4, 0.1, 0, None, BASE, o, None, BASE, 1 << 40, None) == 1
