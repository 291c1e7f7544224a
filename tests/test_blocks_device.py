"""moev_verify_blocks on tensors that are not on the current CUDA device (no GPU: host tensors)."""
import pytest
import torch

import block_ref as R
import paper_2607_12696_b200 as moev
from paper_2607_12696_b200.binding import _Layer, _Linear
from paper_2607_12696_b200.block import verify_blocks

BF16 = torch.bfloat16


class Verifier:  # what verify_blocks takes from a MoeVerifier
    class cfg:
        H = 64
    _h = None

    def _check(self, st):
        raise AssertionError("the call went on")

    def _stream(self):
        return None


class Linear:
    def __init__(self, N, K):
        self._c = _Linear(N, K, moev.W_INT4, 32)
        self.packed = torch.zeros(64, dtype=torch.uint8)
        self._args = (0, self.packed.data_ptr(), 0, -1)


def test_tensors_elsewhere_are_refused():
    s = R.Setup([5], [3], 16, 1, 2, 64, seed=0, spare=0)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    cache = moev.KvCache(s.k, s.v, s.ks, s.vs)
    batch = moev.DraftBatch(i32(s.cu), i32(s.ctx), s.table, 3, 8)
    norm = torch.ones(64, dtype=BF16)
    block = moev.Block(norm, Linear(256, 64), Linear(64, 128), cache, norm, _Layer())
    out = {"y": torch.zeros(3, 64, dtype=BF16), "n_active": torch.zeros(1, dtype=torch.int32)}
    with pytest.raises(moev.MoevError, match="current CUDA device"):
        verify_blocks(Verifier(), [block], batch, torch.zeros(3, 64, dtype=BF16), 2, [out])


def test_every_output_is_looked_at():
    """A diagnostic output on another device than the rest (here: without storage)."""
    s = R.Setup([5], [3], 16, 1, 2, 64, seed=0, spare=0)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    block = moev.Block(torch.ones(64, dtype=BF16), Linear(256, 64), Linear(64, 128), moev.KvCache(s.k, s.v, s.ks, s.vs), torch.ones(64, dtype=BF16), _Layer())
    for name in ("topk_ids", "topk_w", "union_ids", "offsets", "perm"):
        out = {"y": torch.zeros(3, 64, dtype=BF16), "n_active": torch.zeros(1, dtype=torch.int32), name: torch.zeros(64, dtype=torch.int32, device="meta")}
        with pytest.raises(moev.MoevError, match="different devices"):
            verify_blocks(Verifier(), [block], moev.DraftBatch(i32(s.cu), i32(s.ctx), s.table, 3, 8), torch.zeros(3, 64, dtype=BF16), 2, [out])
