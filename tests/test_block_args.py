"""Refusals of the operators around the MoE layer, and their float64 forms against brute force (no GPU)."""
import ctypes as C
import math

import pytest
import torch

import block_ref as R
import paper_2607_12696_b200 as moev
from paper_2607_12696_b200.binding import _DraftBatch, _KvCache, _Linear, _Norm

L = moev.lib()
BUF = (C.c_uint8 * (1 << 16))()
BASE = (C.addressof(BUF) + 255) & ~255  # host memory: every call below is refused before it is looked at


def norm(**kw):
    p = dict(n=2, H=256, afmt=1, wfmt=1, eps=1e-6, act_quant=0, x=BASE, w=BASE, y=BASE, x_stride=256, y_stride=256)
    p.update(kw)
    return L.moev_add_rmsnorm(C.byref(_Norm(**p)), None)


@pytest.mark.parametrize("bad", [dict(H=0), dict(H=32769), dict(n=-1), dict(afmt=2), dict(wfmt=-1), dict(eps=-1.0), dict(eps=math.nan),
                                 dict(act_quant=3), dict(act_quant=1), dict(codes=BASE), dict(act_quant=1, codes=BASE, codes_stride=256), dict(x=None),
                                 dict(w=None), dict(y=None), dict(x_stride=255), dict(y_stride=100), dict(x=BASE + 1), dict(w=BASE + 1),
                                 dict(residual=BASE, residual_stride=8), dict(afmt=0, x=BASE + 2),
                                 dict(act_quant=2, codes=BASE, codes_stride=128, scales=BASE)])
def test_norm_refuses(bad):
    assert norm(**bad) == 1


def test_nothing_to_do_is_fine():
    assert norm(n=0) == 0
    assert L.moev_linear_w4(C.byref(_Linear(16, 64, 4, 32)), BASE, None, BASE, 64, 0, BASE, 16, 1, None) == 0


@pytest.mark.parametrize("N,K,wfmt,group", [(0, 64, 4, 32), (16, 0, 4, 32), (16, 48, 4, 32), (16, 64, 4, 16), (16, 96, 4, 64), (16, 64, 3, 64),
                                            (16, 64, 2, 32), (16, 64, 4, 256)])
def test_linear_refuses_descriptions(N, K, wfmt, group):
    p = C.byref(_Linear(N, K, wfmt, group))
    assert L.moev_w4_packed_bytes(p) == 0
    assert L.moev_w4_pack(p, BASE, BASE, BASE, None) == 1
    assert L.moev_linear_w4(p, BASE, None, BASE, K, 1, BASE, N, 1, None) == 1


def test_linear_refuses_calls():
    p = C.byref(_Linear(16, 64, 4, 32))
    call = lambda **k: L.moev_linear_w4(p, *[{**dict(w=BASE, b=None, x=BASE, xs=64, n=2, y=BASE, ys=16, f=1, st=None), **k}[a]  # noqa: E731
                                             for a in ("w", "b", "x", "xs", "n", "y", "ys", "f", "st")])
    for bad in (dict(w=None), dict(w=BASE + 8), dict(x=None), dict(x=BASE + 1), dict(y=None), dict(xs=63), dict(ys=15), dict(n=-1), dict(f=2),
                dict(f=0, y=BASE + 2), dict(b=BASE + 1)):
        assert call(**bad) == 1


def test_packed_size_is_codes_and_scales_in_whole_tiles_and_a_tail():
    for N, K, wfmt, group, scale in ((16, 128, 4, 128, 32), (17, 160, 4, 32, 128), (1, 64, 3, 32, 64), (33, 192, 4, 64, 64)):
        tiles, chunks = -(-N // 16), -(-K // 128)
        assert L.moev_w4_packed_bytes(C.byref(_Linear(N, K, wfmt, group))) == tiles * chunks * (1024 + scale) + 4096


def cache(**kw):
    return _KvCache(**{**dict(n_pages=4, page=16, n_kv_heads=2, head_dim=64, k=BASE, v=BASE, k_scale=BASE, v_scale=BASE), **kw})


def batch(**kw):
    return _DraftBatch(**{**dict(n_seq=1, n_tokens=3, max_drafts=3, max_len=40, table_cols=3, cu=BASE, ctx_len=BASE, page_table=BASE), **kw})


BAD_CACHE = [dict(n_pages=0), dict(page=8), dict(page=48), dict(page=256), dict(n_kv_heads=0), dict(head_dim=96), dict(k=None), dict(v=BASE + 8),
             dict(k_scale=None), dict(v_scale=BASE + 2)]
BAD_BATCH = [dict(n_seq=-1), dict(n_seq=70000), dict(n_tokens=-1), dict(max_drafts=0), dict(max_len=2), dict(table_cols=0), dict(cu=None),
             dict(ctx_len=None), dict(page_table=None), dict(parent=BASE, max_drafts=1025, max_len=2000), dict(max_len=(1 << 30) + 1)]


@pytest.mark.parametrize("bc,bb", [(b, {}) for b in BAD_CACHE] + [({}, b) for b in BAD_BATCH])
def test_cache_calls_refuse_caches_and_batches(bc, bb):
    c, b = C.byref(cache(**bc)), C.byref(batch(**bb))
    assert L.moev_cache_append(c, b, BASE, 128, BASE, 128, None, 0, None, 0, 0, None, 0, None) == 1
    assert L.moev_cache_attend(c, b, BASE, 256, 4, 0.1, 0, None, BASE, 256, None, BASE, 1 << 40, None) == 1
    assert L.moev_cache_attend_workspace(c, b, 4, 0) == 0


def test_cache_calls_refuse_arguments():
    c, b = C.byref(cache()), C.byref(batch())
    app = lambda **k: L.moev_cache_append(c, b, *[{**dict(k=BASE, ks=128, v=BASE, vs=128, r=None, rr=0, q=None, qs=0, h=0, o=None, os=0, st=None), **k}[a]  # noqa: E731
                                                  for a in ("k", "ks", "v", "vs", "r", "rr", "q", "qs", "h", "o", "os", "st")])
    for bad in (dict(k=None), dict(v=BASE + 2), dict(ks=127), dict(ks=132), dict(vs=120), dict(r=BASE, rr=0), dict(r=BASE + 4, rr=9),
                dict(q=BASE, qs=256, h=4), dict(q=BASE, qs=256, h=3, o=BASE, os=256), dict(q=BASE, qs=255, h=4, o=BASE, os=256),
                dict(q=BASE, qs=256, h=4, o=BASE + 2, os=256), dict(q=BASE, qs=128, h=4, o=BASE, os=256)):
        assert app(**bad) == 1
    att = lambda **k: L.moev_cache_attend(c, b, *[{**dict(q=BASE, qs=256, h=4, s=0.1, w=0, si=None, o=BASE, os=256, l=None, ws=BASE, n=1 << 40, st=None),  # noqa: E731
                                                   **k}[a] for a in ("q", "qs", "h", "s", "w", "si", "o", "os", "l", "ws", "n", "st")])
    for bad in (dict(q=None), dict(q=BASE + 8), dict(qs=252), dict(qs=128), dict(h=3), dict(h=0), dict(s=0.0), dict(s=-1.0), dict(s=math.nan),
                dict(s=math.inf), dict(w=-1), dict(o=None), dict(os=250), dict(l=BASE + 1), dict(si=BASE + 1)):
        assert att(**bad) == 1


def test_attend_refuses_a_small_workspace():
    c, b = C.byref(cache(n_pages=4000)), C.byref(batch(max_len=40000, table_cols=2500))
    size = L.moev_cache_attend_workspace(c, b, 4, 0)
    # sequences + 1 entries of 8 bytes, and a tile of 16 rows of D + 2 floats per CTA and per (sequence, head, rows) segment
    assert size > 0 and (size - 16) % (16 * 66 * 4) == 0
    for ws, n in ((None, size), (BASE + 8, size), (BASE, size - 1)):
        assert L.moev_cache_attend(c, b, BASE, 256, 4, 0.1, 0, None, BASE, 256, None, ws, n, None) == 1


def test_python_layer_names_what_does_not_fit():
    t = torch.zeros
    with pytest.raises(moev.MoevError, match="codes"):
        moev.W4Linear(t(4, 32), t(4, 2), moev.W_INT4, 32)
    with pytest.raises(moev.MoevError, match="no 4-bit linear"):
        moev.W4Linear(t(4, 24, dtype=torch.uint8), t(4, 2), moev.W_INT4, 32)
    with pytest.raises(moev.MoevError, match="scales"):
        moev.W4Linear(t(4, 32, dtype=torch.uint8), t(4, 2), moev.W_INT4, 32)
    with pytest.raises(moev.MoevError, match="x: expected"):
        moev.add_rmsnorm(t(4, 8, dtype=torch.float16), t(8), {})
    with pytest.raises(moev.MoevError, match="weight"):
        moev.add_rmsnorm(t(4, 8), t(9), {"y": t(4, 8)})
    with pytest.raises(moev.MoevError, match="y: expected"):
        moev.add_rmsnorm(t(4, 8), t(8), {"y": t(4, 7)})
    with pytest.raises(moev.MoevError, match="contiguous"):
        moev.add_rmsnorm(t(8, 4).T, t(8), {"y": t(4, 8)})
    with pytest.raises(moev.MoevError, match="current CUDA device"):
        moev.add_rmsnorm(t(4, 8), t(8), {"y": t(4, 8)})
    with pytest.raises(moev.MoevError, match="pages of"):
        moev.KvCache.empty(3, 24, 1, 64, device="cpu")
    with pytest.raises(moev.MoevError, match="disagree"):
        i = lambda *s: t(*s, dtype=torch.int32)  # noqa: E731
        moev.DraftBatch(i(3), i(3), i(3, 2), 1, 4)
    kv = moev.KvCache.empty(3, 16, 2, 64, device="cpu")
    d = moev.DraftBatch(i(4), i(3), i(3, 2), 1, 4, parent=i(2))
    with pytest.raises(moev.MoevError, match="parent has"):
        moev.cache_append(kv, d, t(3, 2, 64, dtype=torch.bfloat16), t(3, 2, 64, dtype=torch.bfloat16))
    with pytest.raises(moev.MoevError, match="k: expected"):
        moev.cache_append(kv, d, t(2, 3, 64, dtype=torch.bfloat16), t(2, 2, 64, dtype=torch.bfloat16))


def test_reference_attention_is_softmax_over_what_a_draft_sees():
    s = R.Setup([5, 0], [4, 3], 16, 1, 1, 64, True, seed=2)
    out, lse = s.attend()[:2]
    paths = R.ancestors(s.parents[0])
    assert [p[-1] for p in paths] == [0, 1, 2, 3]
    i = 3
    kv = [(c, j) for c, j in [(j // 16, j % 16) for j in list(range(5)) + [5 + a for a in paths[i]]]]
    num, den = torch.zeros(64, dtype=torch.float64), 0.0
    for col, off in kv:
        p = int(s.table[0, col])
        w = math.exp(float((s.k[p, 0, off].double() * s.ks[p, 0]) @ s.q[i, 0].double()) / 8)
        num, den = num + w * s.v[p, 0, :, off].double() * s.vs[p, 0], den + w
    assert torch.allclose(out[i, 0], num / den) and abs(float(lse[i, 0]) - math.log(den)) < 1e-9


def test_reference_scale_is_the_smallest_power_of_two():
    for a in (448.0, 449.0, 1.0, 7.0, 7.001, 3e-20, 1e30):
        s = R.pow2_scale(a)
        assert 448 * s >= a > 224 * s and math.frexp(s)[0] == 0.5
