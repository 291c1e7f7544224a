"""The operators on empty tensors and batches, as they come from torch; single rows and sequences beside them."""
import pytest
import torch

import paper_2607_12696_b200 as moev

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_no_rows():
    dev = dict(device="cuda")
    w = torch.ones(256, dtype=BF16, **dev)
    for quant in (0, 1, 2):
        x = torch.empty(0, 256, dtype=BF16, **dev)
        out = {"y": torch.empty_like(x), "residual": torch.empty_like(x)}
        if quant:
            out.update(codes=torch.empty(0, 256, dtype=torch.uint8, **dev), scales=torch.empty(0, 2, **dev))
        moev.add_rmsnorm(x, w, out, residual=x, act_quant=quant)
    lin = moev.W4Linear(torch.zeros(48, 128, dtype=torch.uint8, **dev), torch.ones(48, 8, dtype=BF16, **dev))
    assert lin(x).shape == (0, 48)
    torch.cuda.synchronize()


@pytest.mark.parametrize("n_seq", [0, 3])
def test_no_drafts(n_seq):
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = moev.KvCache.empty(4, 16, 2, 64)
    for parent in (None, i32(0)):
        batch = moev.DraftBatch(i32(n_seq + 1), i32(n_seq), i32(n_seq, 2), 4, 32, parent, i32(1))
        k = torch.empty(0, 2, 64, dtype=BF16, device="cuda")
        for q in (torch.empty(0, 8, 64, dtype=BF16, device="cuda"), torch.empty(0, 512, dtype=BF16, device="cuda")):
            moev.cache_append(cache, batch, k, k, q=q)
            out = moev.cache_attend(cache, batch, q, lse=torch.empty(0, 8, device="cuda"), sinks=torch.zeros(8, device="cuda"))
            assert out.shape == q.shape
    torch.cuda.synchronize()
    assert not cache.k.any() and int(batch.status) == 0
    with pytest.raises(moev.MoevError):
        moev.cache_attend(cache, batch, torch.empty(0, 8, 63, dtype=BF16, device="cuda"))
