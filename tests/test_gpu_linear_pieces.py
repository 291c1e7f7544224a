"""The 4-bit linear layer with x staged piece by piece, in every format; NaN and infinity in x."""
import pytest
import torch

import block_ref as R
import paper_2607_12696_b200 as moev

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
FORMATS = [(False, 32), (False, 64), (False, 128), (True, 32)]


def weight(N, K, mx, group, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8, device="cuda")
    if mx:
        scales = torch.randint(112, 124, (N, K // 32), generator=g, dtype=torch.uint8, device="cuda")
    else:
        scales = (torch.rand(N, K // group, generator=g, device="cuda") * 0.02 + 0.001).to(BF16)
    return codes, scales, moev.W_MXFP4 if mx else moev.W_INT4


def case(n, N, K, mx, group, yd, bias, off=0, seed=5):
    codes, scales, fmt = weight(N, K, mx, group, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    b = torch.randn(N, generator=g, device="cuda") if bias else None
    x = torch.randn(n, K + 8, generator=g, device="cuda").to(BF16)[:, off:off + K]
    y = torch.full((n, N + 3), 7.0, dtype=yd, device="cuda")
    moev.W4Linear(codes, scales, fmt, group, b)(x, y[:, :N])
    w = R.w4_weight(codes, scales, mx, group)
    ref, mass = x.double() @ w.T, x.double().abs() @ w.abs().T
    if bias:
        ref, mass = ref + b.double(), mass + b.double().abs()
    # exact products, K + 8 binary32 additions (the adder may truncate), one rounding of y; MXFP4 takes x off by at most 2^-40
    # of its chunk's largest element
    tol = R.HALF[yd] * (1 + 2.0 ** -7) * ref.abs() + (K + 8) * 2.0 ** -23 * mass
    if mx:
        tol = tol + 2.0 ** -40 * x.double().abs().amax(1, keepdim=True) * w.abs().sum(1)
    off_by = ((y[:, :N].double() - ref).abs() / tol).max()
    assert off_by <= 1, f"{float(off_by):.3g} times the tolerance"
    assert (y[:, N:] == 7).all()


@pytest.mark.parametrize("mx,group", FORMATS)
@pytest.mark.parametrize("n,N,K", [(32, 2880, 4096), (64, 5120, 2880), (32, 1000, 8192), (45, 3000, 7168), (20, 40000, 4096), (17, 100, 12288), (128, 640, 5760),
                                   (16, 500, 16384), (8, 300, 32768)])
def test_pieces(mx, group, n, N, K):
    if K % group:
        K = K // group * group
    case(n, N, K, mx, group, BF16, True)


@pytest.mark.parametrize("mx,group,K", [(False, 32, 7200), (False, 64, 7232), (False, 32, 4128), (True, 32, 7200), (True, 32, 4128), (True, 32, 8160)])
def test_pieces_with_a_tail_and_rows_off_any_boundary(mx, group, K):
    """K that ends inside a chunk of the last piece; a partial last pass of rows."""
    case(32, 333, K, mx, group, F32, True)
    case(45, 2000, K, mx, group, F32, False, off=1)
    case(33, 17, K, mx, group, BF16, True, off=3)


@pytest.mark.parametrize("mx,group", FORMATS)
@pytest.mark.parametrize("n,K", [(3, 256), (20, 256), (32, 8192)])
def test_values_that_are_not_finite(mx, group, n, K):
    """Rows with a NaN or an infinity have what the products say; the other rows are as without them."""
    N = 48
    codes, scales, fmt = weight(N, K, mx, group, 9)
    x = torch.randn(n, K, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    lin = moev.W4Linear(codes, scales, fmt, group)
    clean = lin(x)
    w = R.w4_weight(codes, scales, mx, group)
    for at in (0, 17, 130, K - 1):
        for bad in (float("inf"), -float("inf"), float("nan")):
            z = x.clone()
            z[1, at] = bad
            y = lin(z)
            keep = torch.arange(n) != 1
            assert torch.equal(y[keep.cuda()], clean[keep.cuda()])
            want = bad * w[:, at]  # infinite by the weight's sign, NaN where the weight is zero
            assert torch.equal(y[1].isnan(), want.isnan())
            assert torch.equal(y[1].float().nan_to_num(nan=0.0, posinf=1.0, neginf=-1.0), want.sign().nan_to_num(nan=0.0).float())


@pytest.mark.parametrize("mx,group", FORMATS)
def test_large_and_small_elements_side_by_side(mx, group):
    """Elements that differ by 2^60 within a chunk, the largest finite value, subnormal rows."""
    N, K = 64, 512
    codes, scales, fmt = weight(N, K, mx, group, 11)
    x = torch.randn(4, K, generator=torch.Generator().manual_seed(2))
    x[0, ::7] *= 2.0 ** 20
    x[1, ::5] *= 2.0 ** -60
    x[2] *= 2.0 ** -120
    x[3, 3] = 2.0 ** 100
    x = x.to(BF16).cuda()
    y = torch.empty(4, N, device="cuda")
    moev.W4Linear(codes, scales, fmt, group)(x, y)
    w = R.w4_weight(codes, scales, mx, group)
    ref, mass = x.double() @ w.T, x.double().abs() @ w.abs().T
    tol = (2.0 ** -24 + (K + 8) * 2.0 ** -23) * mass + 2.0 ** -126
    if mx:
        # an element is off by at most 2^-40 of the largest one of its chunk of 128
        top = x.double().abs().view(4, -1, 128).amax(2).repeat_interleave(128, 1)
        tol = tol + 2.0 ** -40 * top @ w.abs().T
    assert ((y.double() - ref).abs() <= tol).all()
