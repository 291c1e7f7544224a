"""Copies of the objects that keep addresses (no GPU)."""
import copy
import ctypes as C
import pickle

import pytest
import torch

import paper_2607_12696_b200 as moev
from paper_2607_12696_b200.binding import _Linear


def linear(bias):
    w = moev.W4Linear.__new__(moev.W4Linear)  # as its constructor leaves it, without a GPU
    w.N, w.K, w.wfmt, w.group = 16, 64, moev.W_INT4, 32
    w._c = _Linear(16, 64, moev.W_INT4, 32)
    w.bias = torch.arange(16.0) if bias else None
    w.packed = torch.arange(64, dtype=torch.uint8)
    w._args = (C.addressof(w._c), w.packed.data_ptr(), w.bias.data_ptr() if bias else 0, -1)
    return w


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda w: pickle.loads(pickle.dumps(w))])
def test_a_copied_weight_reads_its_own_tensors(how, bias):
    w = linear(bias)
    c = how(w)
    assert c._args == (C.addressof(c._c), c.packed.data_ptr(), c.bias.data_ptr() if bias else 0, -1)
    assert torch.equal(c.packed, w.packed) and (c.N, c.K, c.wfmt, c.group) == (16, 64, moev.W_INT4, 32)
    assert (c._c.N, c._c.K, c._c.wfmt, c._c.group) == (16, 64, moev.W_INT4, 32)


def test_caches_and_batches_are_not_copied_with_stale_addresses():
    kv = moev.KvCache.empty(3, 16, 1, 64, device="cpu")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    for thing in (kv, moev.DraftBatch(i32(2), i32(1), i32(1, 2), 3, 8)):
        with pytest.raises(ValueError):
            copy.deepcopy(thing)
