"""Weights that are rows of a larger tensor, wherever those begin."""
import pytest
import torch

import paper_2607_12696_b200 as moev

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("mx,group", [(False, 32), (False, 64), (False, 128), (True, 32)])
@pytest.mark.parametrize("row0", [1, 3, 5, 16])
def test_rows_of_a_larger_weight(mx, group, row0):
    N, K = 40, 128 * 3
    g = torch.Generator(device="cuda").manual_seed(row0)
    codes = torch.randint(0, 256, (N + row0, K // 2), generator=g, dtype=torch.uint8, device="cuda")
    if mx:
        scales = torch.randint(118, 124, (N + row0, K // 32), generator=g, dtype=torch.uint8, device="cuda")
    else:
        scales = (torch.rand(N + row0, K // group, generator=g, device="cuda") + 0.5).to(BF16)
    fmt = moev.W_MXFP4 if mx else moev.W_INT4
    x = torch.randn(3, K, generator=g, device="cuda").to(BF16)
    want = moev.W4Linear(codes, scales, fmt, group)(x)[:, row0:]
    assert torch.equal(moev.W4Linear(codes[row0:], scales[row0:], fmt, group)(x), want)


def test_codes_off_a_16_byte_boundary():
    N, K = 40, 128
    flat = torch.randint(0, 256, (N * K // 2 + 4,), dtype=torch.uint8, device="cuda")
    codes, scales = flat[4:].view(N, K // 2), torch.ones(N, 4, dtype=BF16, device="cuda")
    x = torch.randn(3, K, device="cuda").to(BF16)
    assert torch.equal(moev.W4Linear(codes, scales)(x), moev.W4Linear(codes.clone(), scales)(x))
