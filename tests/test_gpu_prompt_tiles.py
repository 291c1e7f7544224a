"""Prompt attention in its form of two tiles of rows, at the masks that set its tiles apart, against float64.

The host takes that form where the rows may see more than 700 keys (the smaller of the window and, with key rows of their own, all keys of the
call, else the bound on the tokens) and there are too many CTAs for a cluster to share keys: hence the keys of no sequence and the
empty sequences here."""
import pytest
import torch

import paper_2607_12696_b200 as moev
import prompt_ref as R

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
EMPTY, SPARE = 160, 800


def within(got, want, tol, what):
    got, want = got.double().cpu(), want.cpu()
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(got[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)]), f"{what}: other infinities"
    over = ((got - want).abs() - tol)[~odd]
    assert over.numel() == 0 or float(over.max()) <= 0, f"{what}: off by {float(over.max())} more than it may be"


def starts(counts):
    return [sum(counts[:b]) for b in range(len(counts) + 1)]


def make(n_q, n_k, kv, rep, D, seed=0, empty=EMPTY):
    """q, k, v on the host, offsets with empty sequences behind the others, rows of no sequence behind them."""
    g = torch.Generator().manual_seed(seed)
    cu, cu_k = starts(n_q), starts(n_k)
    q, k, v = (torch.randn(*s, generator=g).to(BF16) for s in ((cu[-1] + 2, kv * rep, D), (cu_k[-1] + SPARE, kv, D), (cu_k[-1] + SPARE, kv, D)))
    return q, k, v, cu + cu[-1:] * empty, cu_k + cu_k[-1:] * empty


def run(q, k, v, cu, cu_k, most, repeats=1, **kw):
    """out and lse, of buffers that held 7; the same bits every time."""
    batch = moev.PromptBatch(torch.tensor(cu, dtype=I32, device="cuda"), most, cu_k=torch.tensor(cu_k, dtype=I32, device="cuda"))
    dev, first = [t.cuda() for t in (q, k, v)], None
    for _ in range(repeats):
        out, lse = torch.full(q.shape, 7.0, dtype=BF16, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
        moev.prompt_attend(batch, *dev, out, lse, **kw)
        assert first is None or (torch.equal(out.view(torch.int16), first[0].view(torch.int16)) and torch.equal(lse.view(I32), first[1].view(I32)))
        first = first or (out, lse)
    return first


def check(q, k, v, cu, cu_k, most, repeats=1, window=0, sinks=None, rows=slice(None)):
    out, lse = run(q, k, v, cu, cu_k, most, repeats, window=window, sinks=None if sinks is None else sinks.cuda())
    want, want_l, tol, tol_l = R.prompt(q, k, v, cu, cu_k, q.shape[2] ** -0.5, window, sinks, torch.full(q.shape, 7.0), torch.full(q.shape[:2], 7.0))
    within(lse[rows], want_l[rows], tol_l[rows], "lse")
    within(out[rows], want[rows], tol[rows], "out")
    return out, lse


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q,n_k,kv,rep", [([257] * 8, [100] * 8, 1, 1), ([300, 20], [100, 900], 1, 1), ([150, 20, 90], [70, 0, 10], 2, 2), ([60], [25], 1, 5),
                                            ([129, 256], [1, 0], 1, 1)])
def test_tile_that_sees_nothing_beside_one_that_does(n_q, n_k, kv, rep, D):
    """Fewer keys than tokens by a tile of rows and more: its outputs are 0 every time, whatever its queries are."""
    check(*make(n_q, n_k, kv, rep, D, seed=rep), 1000, repeats=200)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,kv,rep,window", [(900, 1, 1, 705), (900, 1, 1, 0), (300, 2, 4, 0), (170, 1, 8, 0)])
def test_both_tiles_hide_the_same_values(n, kv, rep, window, D):
    """NaN and infinities in keys that come later, that the window has left behind, and of nobody: both tiles of rows clear the same shared tile of V."""
    q, k, v, cu, cu_k = make([n, 40], [n, 40], kv, rep, D, seed=window)
    for t in (k, v):
        t[n - 20, 0, 3] = torch.nan
        t[n - 5, 0, 40], t[n - 3, 0, 40] = torch.inf, -torch.inf
        t[n + 40:] = torch.nan
    if window:  # rows from 745 on see none of these; rows of the same tiles in front of them do
        for t in (k, v):
            t[20:40:5, 0, 7] = torch.nan
            t[39, 0, 9] = torch.inf
    rows = torch.zeros(q.shape[0], dtype=torch.bool)
    rows[:20], rows[(745 if window else 20):n - 20], rows[n:n + 40] = True, True, True
    check(q, k, v, cu, cu_k, 1000, repeats=50, window=window, rows=rows)


@pytest.mark.parametrize("D", [64, 128])
def test_values_that_one_of_two_tiles_sees_stay(D):
    n = 400
    q, k, v, cu, cu_k = make([n], [n], 1, 1, D, seed=3)
    v[130, 0, 3], v[n - 9, 0, 5], v[n - 7, 0, 6], v[n - 5, 0, 6] = torch.inf, torch.nan, torch.inf, -torch.inf
    check(q, k, v, cu, cu_k, 1000, repeats=50)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q,n_k,kv,rep,window", [([5], [130], 1, 136, 0), ([9], [800], 1, 128, 0), ([30, 1, 17], [200, 400, 17], 1, 5, 0), ([20, 6], [12, 0], 2, 2, 0),
                                                   ([120, 3], [900, 740], 1, 2, 705), ([200], [1100], 1, 3, 705)])
def test_two_tiles_keys_of_their_own_windows_and_sinks(n_q, n_k, kv, rep, window, D):
    q, k, v, cu, cu_k = make(n_q, n_k, kv, rep, D, seed=rep)
    sinks = torch.randn(kv * rep, generator=torch.Generator().manual_seed(1))
    check(q, k, v, cu, cu_k, 1000, window=window, sinks=sinks)
    check(q, k, v, cu, cu_k, 1000, window=window)
