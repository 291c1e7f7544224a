"""Calls with nothing to do (no rows, no sequences): empty tensors have no address, and that is fine.  No GPU: nothing is launched."""
import ctypes as C

import pytest

import paper_2607_12696_b200 as moev
from paper_2607_12696_b200.binding import _DraftBatch, _Linear, _Norm
from test_block_args import BASE, cache

L = moev.lib()


@pytest.mark.parametrize("quant", [0, 1, 2])
def test_norm_of_no_rows(quant):
    assert L.moev_add_rmsnorm(C.byref(_Norm(n=0, H=256, afmt=1, wfmt=1, eps=1e-6, act_quant=quant, w=BASE)), None) == 0
    assert L.moev_add_rmsnorm(C.byref(_Norm(n=0, H=0, afmt=1, wfmt=1, eps=1e-6, act_quant=quant, w=BASE)), None) == 1
    assert L.moev_add_rmsnorm(C.byref(_Norm(n=0, H=256, afmt=1, wfmt=1, eps=1e-6, act_quant=3, w=BASE)), None) == 1


def test_linear_of_no_rows():
    p = C.byref(_Linear(16, 64, 4, 32))
    assert L.moev_linear_w4(p, BASE, None, None, 64, 0, None, 16, 1, None) == 0
    assert L.moev_linear_w4(p, None, None, None, 64, 0, None, 16, 1, None) == 1
    assert L.moev_linear_w4(p, BASE, None, None, 64, 1, None, 16, 1, None) == 1


def test_cache_calls_without_rows_or_sequences():
    c = C.byref(cache())
    for d in (_DraftBatch(n_seq=0, n_tokens=0, max_drafts=3, max_len=40, table_cols=3, cu=BASE),
              _DraftBatch(n_seq=0, n_tokens=0, max_drafts=3, max_len=40, table_cols=3),
              _DraftBatch(n_seq=2, n_tokens=0, max_drafts=3, max_len=40, table_cols=3, cu=BASE, ctx_len=BASE, page_table=BASE)):
        b = C.byref(d)
        assert L.moev_cache_append(c, b, None, 128, None, 128, None, 0, None, 0, 0, None, 0, None) == 0
        assert L.moev_cache_attend(c, b, None, 256, 4, 0.1, 0, None, None, 256, None, None, 0, None) == 0
    b = C.byref(_DraftBatch(n_seq=1, n_tokens=0, max_drafts=3, max_len=40, table_cols=3))  # a sequence needs its numbers
    assert L.moev_cache_append(c, b, None, 128, None, 128, None, 0, None, 0, 0, None, 0, None) == 1
    b = C.byref(_DraftBatch(n_seq=0, n_tokens=3, max_drafts=3, max_len=40, table_cols=3))  # rows have an address
    assert L.moev_cache_append(c, b, None, 128, None, 128, None, 0, None, 0, 0, None, 0, None) == 1
