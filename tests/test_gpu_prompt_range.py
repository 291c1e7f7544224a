"""Prompt attention where later keys outweigh the first ones and values are large: the sums stay inside binary32."""
import pytest
import torch

from test_gpu_prompt_tiles import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [2.0 ** 70, 2.0 ** 107])
@pytest.mark.parametrize("n,empty,most", [(600, 0, 600), (400, 300, 400), (600, 160, 1000)])
def test_large_values_behind_scores_that_grow(n, empty, most, size, D):
    """Scores rise by a few powers of two from tile to tile, 50 in all.  600 keys of less than 6 * 2^107 each (7 standard deviations: 2^2.6), times 2^8, sum up to
    less than 2^(9.3 + 2.6 + 107 + 8) = 2^126.9."""
    q, k, v, cu, cu_k = make([n], [n], 1, 2, D, empty=empty)
    q[:], k[:] = 1, 0
    steps = torch.arange(k.shape[0]).clamp(max=n)[:, None, None] * (50 * 0.6931 / n / D ** 0.5)  # D equal products times D^-1/2
    k[:] = steps.to(torch.bfloat16)
    v[:] = (v.float() * size).to(torch.bfloat16)
    assert float(v.float().abs().max()) < 6 * size
    out, _ = check(q, k, v, cu, cu_k, most)
    assert torch.isfinite(out).all()
