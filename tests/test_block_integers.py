"""Host integers that do not fit the 32 bits of the C entry points: refused, not taken modulo 2^32."""
import pytest
import torch

import paper_2607_12696_b200 as moev
from paper_2607_12696_b200.binding import _Layer
from test_blocks_device import Linear, Verifier

BF16 = torch.bfloat16
BIG = [2 ** 32 + 4, 2 ** 31, -2 ** 31 - 1, 2 ** 64 + 1]
i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731


@pytest.mark.parametrize("n", BIG)
def test_batch_bounds(n):
    for bounds in (dict(max_drafts=n, max_len=8), dict(max_drafts=2, max_len=n)):
        with pytest.raises(moev.MoevError, match="32 bits"):
            moev.DraftBatch(i32(2), i32(1), i32(1, 4), **bounds)


@pytest.mark.parametrize("n", BIG)
def test_window_and_heads(n):
    cache = moev.KvCache.empty(3, 16, 1, 64, device="cpu")
    batch = moev.DraftBatch(i32(2), i32(1), i32(1, 1), 3, 8)
    with pytest.raises(moev.MoevError, match="32 bits"):
        moev.cache_attend_workspace(cache, batch, 2, window=n)
    with pytest.raises(moev.MoevError, match="32 bits"):
        moev.cache_attend_workspace(cache, batch, n)
    norm, hidden = torch.ones(64, dtype=BF16), torch.zeros(3, 64, dtype=BF16)
    out = {"y": torch.zeros(3, 64, dtype=BF16), "n_active": i32(1)}
    with pytest.raises(moev.MoevError, match="32 bits"):
        moev.Block(norm, Linear(256, 64), Linear(64, 128), cache, norm, _Layer(), window=n)._c(64, 2)
    with pytest.raises(moev.MoevError, match="32 bits"):
        moev.block.verify_blocks(Verifier(), [moev.Block(norm, Linear(256, 64), Linear(64, 128), cache, norm, _Layer())], batch, hidden, n, [out])


@pytest.mark.parametrize("n", BIG)
def test_weight_groups(n):
    with pytest.raises(moev.MoevError, match="32 bits|no 4-bit linear"):
        moev.W4Linear(torch.zeros(16, 32, dtype=torch.uint8), torch.zeros(16, 2, dtype=BF16), moev.W_INT4, n)
    with pytest.raises(moev.MoevError, match="32 bits|no 4-bit linear"):
        moev.W4Linear(torch.zeros(16, 32, dtype=torch.uint8), torch.zeros(16, 2, dtype=BF16), n, 32)
