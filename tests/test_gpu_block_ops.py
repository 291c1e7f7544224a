"""The operators around the MoE layer against their float64 forms (tests/block_ref.py).

Tolerances.  A result rounded to a type is off by at most half a step of it (2^-8 of the value for bf16, 2^-4 for a
normal e4m3 code, half of 2^-9 below its normal range); what stands in front of that rounding is binary32:
  norm    a sum of H squares in a tree of fewer than 64 sequential steps, a root, two products: 2^-17 of the value
  linear  exact products, K + 8 additions: (K + 8) 2^-23 sum |x w| (2^-23: the tensor core's adder may truncate)
  attend  a probability, its page's V scale relative to a recent largest one and their product are rounded to f16: 3 2^-11;
          below f16's normal range the smallest half step counts, 2^-25, in units in which the row's largest p is 1 or more
          and the tile's largest V scale is 2^-6 or more: 2^-19 pmax vmax |code| per key (`floor`).  The scores' error (ds, an
          exponent) counts twice, on p and on the sum; binary32 sums over keys and chunks 2^-14:
          (3 2^-11 + 2^-14 + 4 ds) sum p |v| + floor.  q in three e4m3 terms is off by 2^-18 of its row's largest
          element or less: part of ds.  lse: 2 ds + 2^-19 (1 + |lse|)
  append  rotation in binary32: 2^-22 of the two products' magnitudes
"""
import pytest
import torch

import block_ref as R
import paper_2607_12696_b200 as moev

pytestmark = pytest.mark.gpu
BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def close(got, ref, tol, what):
    got, ref = got.double().cpu(), ref.double().cpu()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    off = ((got - ref).abs() - tol.cpu()).max() if got.numel() else -1
    assert off <= 0, f"{what}: beyond the tolerance by {float(off):.3e}"


# ------------------------------------------------------------------ norm

def norm_case(n, H, dt, wdt, residual, quant, pad, seed=1, in_place=False, eps=1e-6, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, H + pad, generator=g) * scale).to(dt).cuda()[:, :H]
    res = (torch.randn(n, H + pad, generator=g) * 3 * scale).to(dt).cuda()[:, :H] if residual else None
    w = (1 + 0.3 * torch.randn(H, generator=g)).to(wdt).cuda()
    s, y_ref = R.rmsnorm(x, w, res, eps)
    total = x.float() + res.float() if residual else x.float()
    out = {"y": torch.full((n, H), 7.0, dtype=dt, device="cuda"), "residual": torch.full((n, H), 7.0, dtype=dt, device="cuda")}
    if in_place:
        out = {"y": x, "residual": res if residual else torch.empty_like(x)}
    if quant:
        out["codes"] = torch.full((n, H), 0x55, dtype=torch.uint8, device="cuda")
        out["scales"] = torch.full((n, -(-H // 128)), 7.0, device="cuda")
    moev.add_rmsnorm(x, w, out, residual=res, eps=eps, act_quant=quant)
    torch.cuda.synchronize()
    assert torch.equal(out["residual"], total.to(dt))
    close(out["y"], y_ref, (R.HALF[dt] * (1 + 2.0 ** -7) + 2.0 ** -17) * y_ref.abs(), "y")
    if quant:
        dec, sc = R.decode(out["codes"]), out["scales"].double().repeat_interleave(128, 1)[:, :H]
        blocks = torch.zeros(n, -(-H // 128) * 128, dtype=torch.float64, device="cuda")
        blocks[:, :H] = y_ref
        amax = blocks.view(n, -1, 128).abs().amax(2)
        want = torch.where(amax > 0, amax / 448, 1.0)
        got = out["scales"].double()
        if quant == 1:
            assert ((got - want).abs() <= 2.0 ** -16 * want).all()
        else:
            m, _ = torch.frexp(got)
            assert (m == 0.5).all()
            assert (got >= want * (1 - 2.0 ** -16)).all() and ((got < 2 * want * (1 + 2.0 ** -16)) | (amax == 0)).all()
        close(dec * sc, y_ref, (2.0 ** -4 + 2.0 ** -16) * y_ref.abs() + 2.0 ** -10 * sc, "codes")


@pytest.mark.parametrize("H", [1, 7, 128, 129, 1000, 2880, 4096, 7168, 16384, 32768])
@pytest.mark.parametrize("dt,wdt", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
def test_norm_sizes(H, dt, wdt):
    for n, residual, quant, pad in ((1, True, 0, 0), (3, False, 1, 0), (5, True, 2, 8), (2, True, 1, 3)):
        norm_case(n, H, dt, wdt, residual, quant, pad)


def test_norm_many_rows_and_in_place():
    norm_case(1537, 704, BF16, BF16, True, 1, 0)
    norm_case(300, 1024, BF16, BF16, True, 2, 0, in_place=True)
    norm_case(33, 4097, F32, F32, True, 0, 5, in_place=True)


def test_norm_zero_rows_tiny_and_huge_values():
    w = torch.ones(256, device="cuda", dtype=BF16)
    x = torch.zeros(4, 256, device="cuda", dtype=BF16)
    x[1] = 1e-30
    x[2] = 1e18
    x[3, 5] = 3.0
    out = {"y": torch.empty_like(x), "codes": torch.empty(4, 256, device="cuda", dtype=F8), "scales": torch.empty(4, 2, device="cuda")}
    moev.add_rmsnorm(x, w, out, eps=1e-6, act_quant=2)
    s, ref = R.rmsnorm(x, w, None, 1e-6)
    close(out["y"], ref, (2.0 ** -8 * (1 + 2.0 ** -7) + 2.0 ** -17) * ref.abs(), "y")
    assert (out["codes"][0].float() == 0).all() and (out["scales"][0] == 1).all() and out["scales"][3, 1] == 1
    x[0, 3] = float("nan")
    moev.add_rmsnorm(x, w, out, eps=1e-6, act_quant=1)
    assert out["y"][0].isnan().all() and out["codes"][0].float().isnan().all() and out["y"][1:].isfinite().all()


# ------------------------------------------------------------------ 4-bit linear

def w4_case(n, N, K, mx, group, yd, bias, seed=3, pad=0, off=0):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    scales = torch.randint(112, 124, (N, K // 32), generator=g, dtype=torch.uint8) if mx else (torch.rand(N, K // group, generator=g) * 0.02 + 0.001).to(BF16)
    b = torch.randn(N, generator=g) if bias else None
    x = torch.randn(n, K + pad, generator=g).to(BF16)[:, off:off + K]
    lin = moev.W4Linear(codes.cuda(), scales.cuda(), moev.W_MXFP4 if mx else moev.W_INT4, group, None if b is None else b.cuda())
    y = torch.full((n, N + pad), 7.0, dtype=yd, device="cuda")
    lin(x.cuda() if not pad else torch.empty(n, K + pad, dtype=BF16, device="cuda")[:, off:off + K].copy_(x), y[:, :N])
    torch.cuda.synchronize()
    w = R.w4_weight(codes, scales, mx, group)
    ref = x.double() @ w.T + (0 if b is None else b.double())
    mass = x.double().abs() @ w.abs().T + (0 if b is None else b.double().abs())
    close(y[:, :N], ref, R.HALF[yd] * ref.abs() * (1 + 2.0 ** -7) + (K + 8) * 2.0 ** -23 * mass, f"n={n} N={N} K={K}")
    assert (y[:, N:] == 7).all()


FORMATS = [(False, 32), (False, 64), (False, 128), (True, 32)]


@pytest.mark.parametrize("mx,group", FORMATS)
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 70])
def test_linear_rows(mx, group, n):
    w4_case(n, 200, 512, mx, group, BF16, True)


@pytest.mark.parametrize("mx,group", FORMATS)
@pytest.mark.parametrize("N,K", [(1, 128), (15, 256), (16, 128), (33, 384), (130, 2176), (700, 4096), (2880, 640)])
def test_linear_shapes(mx, group, N, K):
    w4_case(5, N, K, mx, group, F32, False)
    w4_case(12, N, K, mx, group, BF16, True, pad=8)


@pytest.mark.parametrize("mx,group,K", [(False, 32, 32), (False, 32, 96), (False, 64, 64), (False, 64, 2880), (True, 32, 32), (True, 32, 2080)])
def test_linear_odd_k(mx, group, K):
    w4_case(3, 100, K, mx, group, F32, True)
    w4_case(20, 100, K, mx, group, BF16, False, pad=3, off=1)  # rows of x off any 16-byte boundary


@pytest.mark.parametrize("n,N,K", [(1, 40000, 256), (16, 70001, 128), (32, 1000, 8192), (24, 20000, 4096), (48, 5000, 7168), (16, 6000, 7168)])
def test_linear_large(n, N, K):
    """Several row groups per CTA; x staged whole and piece by piece."""
    w4_case(n, N, K, False, 64, F32, False)


def test_linear_special_values():
    """A NaN or infinity in one row of x stays in that row; zero scales give zeros; rows behind K are not read."""
    N, K = 48, 256
    codes = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, generator=torch.Generator().manual_seed(0)).cuda()
    scales = torch.full((N, K // 32), 0.5, dtype=BF16, device="cuda")
    scales[7] = 0
    x = torch.randn(3, K, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    x[1, 17] = float("nan")
    lin = moev.W4Linear(codes, scales, moev.W_INT4, 32)
    y = lin(x)
    assert y[1].isnan().all() and y[0].isfinite().all() and y[2].isfinite().all() and (y[0, 7] == 0)


# ------------------------------------------------------------------ cache

def device_cache(s):
    c = moev.KvCache(s.k.cuda().contiguous(), s.v.cuda().contiguous(), s.ks.cuda(), s.vs.cuda())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    d = moev.DraftBatch(torch.tensor(s.cu, dtype=torch.int32).cuda(), torch.tensor(s.ctx, dtype=torch.int32).cuda(), s.table.cuda(), s.max_drafts,
                        s.max_len, None if s.parent is None else s.parent.cuda(), status)
    return c, d


def p_tol(mass, ds, floor):
    return (3 * 2.0 ** -11 + 2.0 ** -14 + 4 * ds)[..., None] * mass + floor


def attend_case(s, window=0, sinks=None, scale=None):
    c, d = device_cache(s)
    out = torch.full((s.T, s.heads * s.rep, s.D), 7.0, dtype=BF16, device="cuda")
    lse = torch.full((s.T, s.heads * s.rep), 7.0, device="cuda")
    moev.cache_attend(c, d, s.q.cuda(), out, lse=lse, scale=scale, window=window, sinks=None if sinks is None else sinks.cuda())
    torch.cuda.synchronize()
    assert int(d.status) == 0
    ref, lref, mass, ds, floor = s.attend(window, sinks, scale)
    live = s.cu[-1]
    close(out[:live], ref[:live], R.HALF[BF16] * (1 + 2.0 ** -7) * ref[:live].abs() + p_tol(mass, ds, floor)[:live] + 1e-30, "out")
    close(lse[:live], lref[:live], (2 * ds + 2.0 ** -19 * (1 + lref.abs()))[:live], "lse")
    assert (out[live:] == 7).all() and (lse[live:] == 7).all()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tree", [False, True])
def test_attend_pages(page, D, tree):
    attend_case(R.Setup([0, 1, 63, 64, 200, 5], [1, 3, 5, 0, 4, 6], page, 2, 3, D, tree, seed=page + D).poison())


@pytest.mark.parametrize("rep,n", [(1, 1), (1, 40), (3, 7), (4, 4), (8, 5), (8, 9), (16, 1), (16, 2), (16, 17), (5, 64)])
def test_attend_row_tiles(rep, n):
    """Every arrangement of warps over rows and keys, rows that end inside a tile of 16."""
    for D in (64, 128):
        attend_case(R.Setup([130, 700, 3], [n, 1, n // 2], 64, 2, rep, D, True, seed=rep * 100 + n).poison())


@pytest.mark.parametrize("window", [1, 2, 31, 64, 100, 1000])
@pytest.mark.parametrize("tree", [False, True])
def test_attend_window_and_sinks(window, tree):
    s = R.Setup([0, 5, 64, 333, 900], [4, 9, 1, 33, 12], 32, 2, 4, 64, tree, seed=window).poison()
    attend_case(s, window=window)
    attend_case(s, window=window, sinks=torch.linspace(-3, 6, s.heads * s.rep))


def test_attend_long_context_splits_and_joins():
    attend_case(R.Setup([9000], [2], 128, 1, 8, 128, seed=1).poison())
    attend_case(R.Setup([5000, 40, 2500], [3, 3, 3], 16, 1, 8, 64, True, seed=2).poison(), scale=0.3)


def test_attend_long_chain_and_deep_tree():
    attend_case(R.Setup([37], [300], 64, 1, 2, 64, seed=5).poison())
    s = R.Setup([20, 3], [200, 77], 64, 1, 1, 128, True, seed=6)
    s.parents[0] = R.chain(200)  # deepest possible tree
    s.parent[:200] = torch.tensor(s.parents[0], dtype=torch.int32)
    attend_case(s.poison())
    attend_case(s, window=50)


def test_attend_nan_in_masked_places_stays_there():
    """A NaN value that some drafts see (their own branch) and others do not."""
    s = R.Setup([70], [4], 64, 1, 2, 64, True, seed=9).poison()
    s.parents[0], s.parent[:4] = [-1, 0, -1, 2], torch.tensor([-1, 0, -1, 2], dtype=torch.int32)
    c, d = device_cache(s)
    slot = 70 + 1  # draft 1: seen by itself only
    p = int(s.table[0, slot // 64])
    c.v.view(torch.uint8)[p, 0, 11, slot % 64] = 0x7F
    clean = moev.cache_attend(c, d, s.q.cuda()).clone()
    assert clean[1, :, 11].isnan().all()
    ok = torch.ones_like(clean, dtype=torch.bool)
    ok[1, :, 11] = False
    assert clean[:4][ok[:4]].isfinite().all()
    c.k.view(torch.uint8)[p, 0, slot % 64, 3] = 0x7F
    out = moev.cache_attend(c, d, s.q.cuda())
    assert out[1].isnan().all() and out[[0, 2, 3]].isfinite().all()


def test_attend_scales_far_apart():
    """Pages whose V scales differ by 2^24, the heavy one first and last."""
    for order in (0, 1):
        s = R.Setup([250], [2], 64, 1, 4, 64, seed=12).poison()
        s.vs[s.table[0].long()] = torch.tensor([1.0, 2.0 ** -12, 2.0 ** -24, 2.0 ** -6] if order else [2.0 ** -24, 2.0 ** -12, 1.0, 4.0])[:, None]
        attend_case(s)


def test_attend_extreme_queries():
    s = R.Setup([100], [5], 16, 1, 2, 64, seed=13).poison()
    s.q[0] = 0
    s.q[1] *= 2.0 ** -40
    s.q[2] *= 40
    s.q[3, :, 5] = 1000.0
    attend_case(s)


def append_case(s, rope=True, with_q=True):
    c, d = device_cache(s)
    before_k, before_v = c.k.view(torch.uint8).clone().cpu(), c.v.view(torch.uint8).clone().cpu()
    q, new, kept, ks, vs = s.append(rope)
    q_out = torch.full_like(s.q, 7.0).cuda() if with_q else None
    moev.cache_append(c, d, s.nk.cuda(), s.nv.cuda(), rope=s.rope.cuda() if rope else None, q=s.q.cuda() if with_q else None, q_out=q_out)
    torch.cuda.synchronize()
    assert int(d.status) == 0
    assert torch.equal(c.k_scale.double().cpu(), ks) and torch.equal(c.v_scale.double().cpu(), vs)
    if with_q:
        live = s.cu[-1]
        tol = R.HALF[BF16] * (1 + 2.0 ** -7) * q.abs() + 2.0 ** -20 * s.q.double().abs().amax(-1, keepdim=True)
        close(q_out[:live], q[:live], tol[:live], "q")
        assert (q_out[live:] == 7).all()
    for name, got, before, sc in (("k", c.k, before_k, ks), ("v", c.v, before_v, vs)):
        code = got.view(torch.uint8).cpu()
        if name == "v":
            code, before = code.transpose(2, 3), before.transpose(2, 3)
        expect = before.clone()
        for p, h, fill, ratio in kept[name]:  # kept tokens: code times a power of two, rounded to the nearest code
            expect[p, h, :fill] = (before[p, h, :fill].contiguous().view(F8).float() * ratio).to(F8).view(torch.uint8)
        fresh = ~new[name].isnan()
        if name == "v":
            assert fresh.shape == code.shape
        same = torch.where(fresh, code, expect)
        assert torch.equal(code, same), f"{name}: bytes outside the new tokens"
        val, want = code.contiguous().view(F8).double() * sc[:, :, None, None], new[name]
        tol = (2.0 ** -4 + 2.0 ** -18) * want.abs() + 2.0 ** -10 * sc[:, :, None, None] + 2.0 ** -20
        assert ((val - want).abs() <= tol)[fresh].all(), f"{name}: new tokens"


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tree", [False, True])
def test_append(page, D, tree):
    s = R.Setup([0, 1, 15, 16, 127, 130, 77], [3, 1, 2, 0, 1, 40, page + 3], page, 2, 3, D, tree, seed=page + D)
    append_case(s)
    append_case(s, rope=False, with_q=False)


def test_append_scale_grows_and_stays():
    """A part-full page whose new tokens need more range (old codes shrink), less (scale kept), or are zero."""
    for mag in (2.0 ** -12, 1.0, 2.0 ** 9, 2.0 ** 20, 0.0):
        s = R.Setup([5, 30, 0], [4, 1, 2], 16, 2, 1, 64, seed=3)
        s.nk = (s.nk.float() * mag).to(BF16)
        s.nv = (s.nv.float() * mag).to(BF16)
        append_case(s, rope=False)


def test_append_nan_and_infinity():
    s = R.Setup([16], [2], 16, 1, 1, 64, seed=4)
    s.nk[0, 0, 3], s.nv[1, 0, 7], s.nv[0, 0, 8] = float("nan"), float("inf"), -float("inf")
    c, d = device_cache(s)
    moev.cache_append(c, d, s.nk.cuda(), s.nv.cuda())
    p = int(s.table[0, 1])
    assert c.k[p, 0, 0, 3].float().isnan() and c.k[p, 0, 0].float().isnan().sum() == 1
    assert c.v[p, 0, 7, 1].float() == 448 and c.v[p, 0, 8, 0].float() == -448 and c.v_scale[p, 0].isfinite()


def test_append_then_attend_is_attention_over_the_appended_tokens():
    """A run of the two as they are used: three steps of ragged trees, each accepting some drafts."""
    D, page, heads, rep = 64, 16, 2, 4
    s = R.Setup([3, 40, 0], [5, 2, 7], page, heads, rep, D, True, seed=8, max_len=80)
    c, d = device_cache(s)
    for step in range(3):
        g = torch.Generator().manual_seed(100 + step)
        s.q, s.nk, s.nv = (torch.randn(s.T, h, D, generator=g).to(BF16) for h in (heads * rep, heads, heads))
        d.ctx_len.copy_(torch.tensor(s.ctx, dtype=torch.int32))
        q = moev.cache_append(c, d, s.nk.cuda(), s.nv.cuda(), rope=s.rope.cuda(), q=s.q.cuda())
        out = moev.cache_attend(c, d, q)
        s.k, s.v, s.ks, s.vs, s.q = c.k.cpu(), c.v.cpu(), c.k_scale.cpu(), c.v_scale.cpu(), q.cpu()
        ref, _, mass, ds, floor = s.attend()
        live = s.cu[-1]
        close(out[:live], ref[:live], R.HALF[BF16] * (1 + 2.0 ** -7) * ref[:live].abs() + p_tol(mass, ds, floor)[:live], "out")
        s.ctx = [a + b for a, b in zip(s.ctx, (2, 0, 5))]


def test_rejected_sequences_and_pages_are_reported_and_skipped():
    s = R.Setup([20, 30, 40], [3, 3, 3], 16, 1, 2, 64, seed=10)
    ref = s.attend()[0]
    c, d = device_cache(s)
    d.ctx_len[1] = 1000  # behind max_len
    out = torch.full((s.T, 2, 64), 7.0, dtype=BF16, device="cuda")
    moev.cache_attend(c, d, s.q.cuda(), out)
    assert int(d.status) == 1 and (out[3:6] == 7).all()
    assert (out[:3].double().cpu() - ref[:3]).abs().max() < 0.1 and (out[6:9].double().cpu() - ref[6:9]).abs().max() < 0.1
    before = c.k.view(torch.uint8).clone()
    moev.cache_append(c, d, s.nk.cuda(), s.nv.cuda())
    own = s.table[1].long()
    assert torch.equal(c.k.view(torch.uint8)[own], before[own])
    c, d = device_cache(s)
    d.page_table[0, 0] = 10 ** 6
    d.page_table[2, 1] = -5
    out = moev.cache_attend(c, d, s.q.cuda())
    assert int(d.status) == 2 and out.isfinite().all()
    assert (out[3:6].double().cpu() - ref[3:6]).abs().max() < 0.1
    c, d = device_cache(s)
    moev.cache_append(c, d, s.nk.cuda(), s.nv.cuda(), rope=s.rope[:20].cuda().contiguous())
    assert int(d.status) == 3


def test_captured_and_replayed():
    """A step captured into a graph, replayed with new lengths and tokens, against eager calls; two graphs, one workspace each."""
    s = R.Setup([20, 300], [3, 5], 16, 2, 4, 64, True, seed=21, max_len=400)
    c, d = device_cache(s)
    c2, d2 = device_cache(s)
    w = torch.ones(512, device="cuda", dtype=BF16)
    lin = moev.W4Linear(torch.randint(0, 256, (512, 256), dtype=torch.uint8, device="cuda"), torch.full((512, 16), 0.02, dtype=BF16, device="cuda"))
    x = torch.randn(s.T, 512, device="cuda").to(BF16)
    nk, nv, q = s.nk.cuda(), s.nv.cuda(), s.q.cuda()

    def step(cache, batch, ws):
        n = moev.add_rmsnorm(x, w, {"y": torch.empty_like(x)})["y"]
        y = lin(n)
        qr = moev.cache_append(cache, batch, nk, nv, rope=rope, q=y.view(s.T, 8, 64), q_out=torch.zeros_like(q))
        return moev.cache_attend(cache, batch, qr, workspace=ws)

    rope = s.rope.cuda()
    step(c2, d2, None)
    for t, u in ((c.k, c2.k), (c.v, c2.v), (c.k_scale, c2.k_scale), (c.v_scale, c2.v_scale)):
        t.copy_(u)
    ws = moev.cache_attend_workspace(c, d, 8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(c, d, ws)
    for ctx in ([20, 300], [23, 310], [0, 64]):
        x.copy_(torch.randn(s.T, 512, generator=torch.Generator().manual_seed(sum(ctx))).to(BF16))
        for b in (d, d2):
            b.ctx_len.copy_(torch.tensor(ctx, dtype=torch.int32))
        graph.replay()
        want = step(c2, d2, None)
        torch.cuda.synchronize()
        live = s.cu[-1]
        assert torch.equal(got[:live], want[:live]) and torch.equal(c.k.view(torch.uint8), c2.k.view(torch.uint8))


def test_two_streams_with_a_workspace_each():
    a, b = (R.Setup([700], [4], 64, 2, 8, 128, True, seed=i).poison() for i in (31, 32))
    ca, da = device_cache(a)
    cb, db = device_cache(b)
    qa, qb = a.q.cuda(), b.q.cuda()
    want = moev.cache_attend(ca, da, qa), moev.cache_attend(cb, db, qb)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(10):
        with torch.cuda.stream(s1):
            x = moev.cache_attend(ca, da, qa)
        with torch.cuda.stream(s2):
            y = moev.cache_attend(cb, db, qb)
        outs.append((x, y))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[0]) and torch.equal(y, want[1]) for x, y in outs)
