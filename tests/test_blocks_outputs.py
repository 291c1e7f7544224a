"""moev_verify_blocks: outputs that are too small, of another type or with gaps (no GPU: refused before anything else)."""
import pytest
import torch

import block_ref as R
import paper_2607_12696_b200 as moev
from paper_2607_12696_b200.binding import _Layer
from paper_2607_12696_b200.block import verify_blocks
from test_blocks_device import Linear, Verifier

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
T, H, E, K = 3, 64, 8, 2


class Sized(Verifier):
    class cfg:
        H, E, top_k = H, E, K


def outputs():
    return {"y": torch.zeros(T, H, dtype=BF16), "n_active": torch.zeros(1, dtype=I32), "topk_ids": torch.zeros(T, K, dtype=I32),
            "topk_w": torch.zeros(T, K), "union_ids": torch.zeros(E, dtype=I32), "offsets": torch.zeros(E + 1, dtype=I32), "perm": torch.zeros(T * K, dtype=I32)}


def call(out, **k):
    s = R.Setup([5], [T], 16, 1, 2, 64, seed=0, spare=0)
    i32 = lambda x: torch.tensor(x, dtype=I32)  # noqa: E731
    norm = torch.ones(H, dtype=BF16)
    block = moev.Block(norm, Linear(256, H), Linear(H, 128), moev.KvCache(s.k, s.v, s.ks, s.vs), norm, _Layer())
    verify_blocks(Sized(), [block], moev.DraftBatch(i32(s.cu), i32(s.ctx), s.table, T, 8), torch.zeros(T, H, dtype=BF16), 2, [out], **k)


@pytest.mark.parametrize("name", ["n_active", "topk_ids", "topk_w", "union_ids", "offsets", "perm"])
def test_diagnostics_that_do_not_fit(name):
    good = outputs()[name]
    other = F32 if good.dtype == I32 else I32
    for bad in (good[:-1], good.to(other), torch.zeros(2 * good.numel(), dtype=good.dtype)[::2].view(good.shape) if good.numel() > 1 else good.double()):
        with pytest.raises(moev.MoevError, match=name):
            call({**outputs(), name: bad})


def test_outputs_that_fit_get_as_far_as_the_device():
    for out in (outputs(), {k: outputs()[k] for k in ("y", "n_active")}, {k: torch.cat([t, t]) for k, t in outputs().items()}):
        with pytest.raises(moev.MoevError, match="current CUDA device"):
            call(out)


def test_a_scale_of_zero_is_no_scale():
    with pytest.raises(moev.MoevError, match="scale"):
        call(outputs(), scale=0.0)
