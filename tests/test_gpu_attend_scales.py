"""Attention over pages whose V scales lie far apart, against float64.

A key's contribution is off by one rounding of p * (V scale) to f16, 2^-11 of it, whatever the scales of other pages: the
reference that keeps this product in f16's range is per row and follows the largest product of a key that the row sees and
whose V is not zero.  What falls below f16's normal range is off by at most 2^-25 in units in which that largest product is 8
or more (2^-28 of it), and scales below 2^-48 of the sequence's largest count with 2^-76 of that.  The rest as for all of
attention: a key's score is off by D truncated binary32 additions and by what three e4m3 terms leave of q (2^-18 of the row's
largest element); it counts on the key's own p and, weighted, on the denominator, each at most twice over; sums 2^-14."""
import pytest
import torch

import block_ref as R
import paper_2607_12696_b200 as moev

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def expected(s, window):
    """(out, tolerance) of the sequences' rows."""
    scale = s.D ** -0.5
    out = torch.zeros(s.T, s.heads * s.rep, s.D, dtype=torch.float64)
    tol = torch.zeros_like(out)
    for b, (c, n) in enumerate(zip(s.ctx, s.cnt)):
        pages = s.table[b, :-(-(c + n) // s.page)].long()
        k = (s.k[pages].double() * s.ks[pages].double()[..., None, None]).permute(1, 0, 2, 3).reshape(s.heads, -1, s.D)
        code = s.v[pages].double().permute(1, 0, 3, 2).reshape(s.heads, -1, s.D)
        vs = s.vs[pages].double().T.repeat_interleave(s.page, 1)
        for i, path in enumerate(R.ancestors(s.parents[b])):
            at = c + len(path) - 1
            keys = [j for j in range(max(0, at - window + 1) if window else 0, c)] + [c + j for j in (path[-window:] if window else path)]
            for hq in range(s.heads * s.rep):
                h, row = hq // s.rep, s.cu[b] + i
                kk, cc, sc = k[h][keys], code[h][keys], vs[h][keys]
                q = s.q[row, hq].double()
                p = torch.softmax(kk @ q * scale, 0)
                ds = scale * (s.D * 2.0 ** -23 * (kk.abs() @ q.abs()) + 2.0 ** -18 * q.abs().max() * kk.abs().sum(1))
                off = 2.0 ** -11 + 2.0 ** -14 + 2 * (ds + (p * ds).sum())
                w = p * sc
                largest = w[cc.abs().amax(1) > 0].max() if cc.any() else 0.0
                floor = (2.0 ** -28 * largest + 2.0 ** -76 * p.max() * vs[h, :c + n].max()) * cc.abs().sum(0)
                out[row, hq] = w @ cc
                tol[row, hq] = R.HALF[BF16] * (1 + 2.0 ** -7) * out[row, hq].abs() + (off * w) @ cc.abs() + floor
    return out, tol


def check(s, window=0):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    cache = moev.KvCache(s.k.cuda().contiguous(), s.v.cuda().contiguous(), s.ks.cuda(), s.vs.cuda())
    batch = moev.DraftBatch(i32(s.cu), i32(s.ctx), s.table.cuda(), s.max_drafts, s.max_len, None if s.parent is None else s.parent.cuda())
    got = moev.cache_attend(cache, batch, s.q.cuda(), window=window).double().cpu()
    ref, tol = expected(s, window)
    live = s.cu[-1]
    assert got[:live].isfinite().all()
    worst = ((got - ref).abs() / tol.clamp(min=1e-300))[:live].max()
    assert worst <= 1, f"{float(worst):.3g} times the tolerance"


ROWS = [(1, 1), (4, 8), (4, 13), (8, 16)]  # drafts, query heads per kv head: every size of a row tile


def spread(s, *exponents):
    """V scales 2^e of the columns of every sequence's table, the last one for all that follow."""
    for b in range(len(s.ctx)):
        for col in range(s.cols):
            s.vs[s.table[b, col].long()] = 2.0 ** exponents[min(col, len(exponents) - 1)]


@pytest.mark.parametrize("n,rep", ROWS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ratio", [-12, -20, -26, -40])
def test_a_page_outside_the_window_does_not_count(n, rep, D, ratio):
    """Keys 0..15 are in the tile and in no window."""
    s = R.Setup([40], [n], 16, 1, rep, D, True, seed=3 + n).poison()
    spread(s, 0, ratio)
    check(s, window=9)


@pytest.mark.parametrize("n,rep", ROWS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ratio", [-16, -20, -26, -60])
@pytest.mark.parametrize("col", [0, 1, 7])
def test_a_page_without_weight_does_not_count(n, rep, D, ratio, col):
    """One page with the largest V scale, in the first tile or the last, whose scores are far below the others'."""
    s = R.Setup([200 if col < 7 else 258], [n], 32, 1, rep, D, seed=5 + n).poison()
    q = s.q.float()
    q[..., 0] = 4.0
    s.q = q.to(BF16)
    heavy = s.table[0, col].long()
    k = s.k.view(torch.uint8).clone()
    k[heavy] = 0
    k[heavy, :, :, 0] = 0xFE  # -448
    s.k = k.view(torch.float8_e4m3fn)
    s.ks[heavy] = 1.0
    spread(s, ratio)
    s.vs[heavy] = 1.0
    check(s)


@pytest.mark.parametrize("n,rep", ROWS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ratio", [-16, -20, -26, -40])
@pytest.mark.parametrize("col", [0, 2, 5])
def test_zero_values_do_not_count(n, rep, D, ratio, col):
    """A page of zeros keeps the scale 1, whatever the values of others; its keys take part in the denominator."""
    s = R.Setup([200], [n], 32, 1, rep, D, True, seed=7 + n).poison()
    spread(s, ratio)
    zero = s.table[0, col].long()
    v = s.v.view(torch.uint8).clone()
    v[zero] = torch.where(torch.rand(v[zero].shape, generator=torch.Generator().manual_seed(1)) < 0.5, 0, 0x80).to(torch.uint8)  # of either sign
    s.v = v.view(torch.float8_e4m3fn)
    s.vs[zero] = 1.0
    check(s)


@pytest.mark.parametrize("n,rep", ROWS)
@pytest.mark.parametrize("exponents", [(0, -30), (-30, 0), (-90, 20, -10), (20, -90, -10), (-90, -20, 60), (3, -5, 8, -12, 0, 2, -9)])
def test_scales_of_every_order(n, rep, exponents):
    """Growing and falling scales over several tiles and, in a long context, several parts."""
    for ctx, page in (([300, 150], 128), ([2500], 64)):
        s = R.Setup(ctx, [n] * len(ctx), page, 1, rep, 64, seed=11 + n).poison()
        spread(s, *exponents)
        check(s)


@pytest.mark.parametrize("n,rep", ROWS)
def test_scales_that_are_no_powers_of_two(n, rep):
    s = R.Setup([300], [n], 32, 2, rep, 64, True, seed=13).poison()
    s.vs = s.vs * (1 + torch.rand(s.vs.shape, generator=torch.Generator().manual_seed(2)))
    s.ks = s.ks * (1 + torch.rand(s.ks.shape, generator=torch.Generator().manual_seed(3)))
    check(s)
