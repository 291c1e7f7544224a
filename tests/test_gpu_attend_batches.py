"""Attention over many sequences: the work split of more than 32 (a scan over the whole CTA, several sequences per thread
behind one per thread), empty and rejected ones among them, segments that are split and segments dealt out whole; and queries
that are not finite."""
import pytest
import torch

import block_ref as R
import paper_2607_12696_b200 as moev

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def device_batch(s):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    cache = moev.KvCache(s.k.cuda().contiguous(), s.v.cuda().contiguous(), s.ks.cuda(), s.vs.cuda())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    return cache, moev.DraftBatch(i32(s.cu), i32(s.ctx), s.table.cuda(), s.max_drafts, s.max_len, None if s.parent is None else s.parent.cuda(), status)


def check(s, window=0, rejected=()):
    cache, batch = device_batch(s)
    for b in rejected:
        batch.ctx_len[b] = s.max_len + 1
    out = torch.full((s.T, s.heads * s.rep, s.D), 7.0, dtype=BF16, device="cuda")
    lse = torch.full((s.T, s.heads * s.rep), 7.0, device="cuda")
    moev.cache_attend(cache, batch, s.q.cuda(), out, lse=lse, window=window)
    torch.cuda.synchronize()
    assert int(batch.status) == (1 if rejected else 0)
    ref, lref, mass, ds, floor = s.attend(window)
    live = torch.ones(s.T, dtype=torch.bool)
    live[s.cu[-1]:] = False
    for b in rejected:
        live[s.cu[b]:s.cu[b + 1]] = False
    # one f16 rounding of p times the page's scale, binary32 sums, the scores' error on p and on the sum
    tol = R.HALF[BF16] * (1 + 2.0 ** -7) * ref.abs() + (2.0 ** -11 + 2.0 ** -14 + 4 * ds)[..., None] * mass + floor + 1e-30
    got = out.double().cpu()
    assert got[live].isfinite().all()
    assert ((got - ref).abs() <= tol)[live].all()
    assert ((lse.double().cpu() - lref).abs() <= 2 * ds + 2.0 ** -19 * (1 + lref.abs()))[live].all()
    assert (out.cpu()[~live] == 7).all() and (lse.cpu()[~live] == 7).all()


def lengths(n, longest, seed, drafts):
    g = torch.Generator().manual_seed(seed)
    ctx = torch.randint(0, longest + 1, (n,), generator=g).tolist()
    cnt = torch.randint(0, drafts + 1, (n,), generator=g).tolist()
    ctx[n // 2], cnt[0], cnt[-1] = longest, drafts, 1
    return ctx, cnt


@pytest.mark.parametrize("n", [31, 32, 33, 64, 100, 321, 577, 700])
@pytest.mark.parametrize("rep,drafts", [(2, 3), (4, 7), (5, 11), (16, 6)])
def test_many_sequences(n, rep, drafts):
    if rep * drafts > 64 and n > 400:
        drafts = 5  # the reference takes a loop per row
    ctx, cnt = lengths(n, 40, n, drafts)
    s = R.Setup(ctx, cnt, 16, 1, rep, 64, True, seed=n + rep).poison()
    check(s)  # a tile or less: dealt out whole
    check(s, rejected=(1, n - 2))


@pytest.mark.parametrize("n", [33, 100, 400])
@pytest.mark.parametrize("rep,drafts,tree", [(2, 2, False), (4, 8, True), (8, 6, True), (16, 5, False)])
def test_many_sequences_that_are_split(n, rep, drafts, tree):
    """Bounds of more than four tiles: runs of tiles that begin and end inside sequences."""
    ctx, cnt = lengths(n, 70, 3 * n, min(drafts, 3) if n > 100 else drafts)
    ctx[3], ctx[n - 3] = 1500, 700
    cnt[3], cnt[n - 3] = drafts, 1
    s = R.Setup(ctx, cnt, 64, 1, rep, 64, tree, seed=n + rep).poison()
    check(s)
    check(s, rejected=(2, 5, n - 1))
    check(s, window=600)


def test_all_sequences_empty_or_rejected():
    for n in (3, 40):
        s = R.Setup([20] * n, [0] * (n - 1) + [2], 16, 1, 2, 64, seed=1).poison()
        check(s, rejected=(n - 1,))


def test_queries_that_are_not_finite():
    """A row with a NaN or an infinity in q has NaN outputs (inf - inf in its softmax); other rows of its tile do not change."""
    for n, rep in ((1, 2), (4, 8), (4, 13), (8, 16)):
        s = R.Setup([200], [n], 32, 1, rep, 64, seed=n).poison()
        cache, batch = device_batch(s)
        clean = moev.cache_attend(cache, batch, s.q.cuda())[:n].clone()
        for bad in (float("nan"), float("inf"), -float("inf")):
            for row, head in ((0, 0), (n - 1, rep - 1)):
                q = s.q.clone()
                q[row, head, 5] = bad
                got = moev.cache_attend(cache, batch, q.cuda())[:n]
                ok = torch.ones(n, rep, dtype=torch.bool)
                ok[row, head] = False
                assert got[row, head].isnan().all()
                assert torch.equal(got[ok.cuda()], clean[ok.cuda()])
            q = s.q.clone()
            q[0, 1] = bad
            assert moev.cache_attend(cache, batch, q.cuda())[0, 1].isnan().all()
