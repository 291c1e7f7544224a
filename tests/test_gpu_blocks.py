"""moev_verify_blocks: decoder blocks of a verification pass (norm, 4-bit projections, cached tree attention, MoE layer).

Against the same steps called one by one (the same kernels; only the order of the MoE layer's fp32 additions may
differ), and the attention half of a block against its float64 form."""
import numpy as np
import pytest
import torch

import block_ref as R
import paper_2607_12696_b200 as moev
import synth
from gpu_common import device_layer, gcfg
from helpers import small_shape

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def linear(N, K, mx, seed, bias):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    if mx:
        scales = torch.randint(118, 121, (N, K // 32), generator=g, dtype=torch.uint8)
        fmt, group = moev.W_MXFP4, 32
    else:
        scales = (torch.rand(N, K // 32, generator=g) * 0.006 + 0.002).to(BF16)
        fmt, group = moev.W_INT4, 32
    b = torch.randn(N, generator=g) * 0.1 if bias else None
    return moev.W4Linear(codes.cuda(), scales.cuda(), fmt, group, None if b is None else b.cuda()), R.w4_weight(codes, scales, mx, group), b


class Model:
    def __init__(self, n_blocks, s, base="gptoss", seed=0, **dims):
        self.shape = small_shape(base, **dims)
        H, D, heads, rep = self.shape.H, s.D, s.heads, s.rep
        self.s, self.T, self.n_heads = s, s.T, heads * rep
        self.v = moev.MoeVerifier(gcfg(self.shape, s.T))
        g = torch.Generator().manual_seed(seed)
        self.blocks, self.weights, self.keep = [], [], []
        for l in range(n_blocks):
            w = synth.make_expert_weights(self.shape, layer=l, device="cuda")
            wr, _ = synth.make_iid_routing(self.shape, s.T, layer=l, device="cuda")
            layer, keep = device_layer(wr, w)
            qkv, wq, bq = linear((heads * rep + 2 * heads) * D, H, l % 2 == 0, 10 * seed + l, True)
            o, wo, bo = linear(H, heads * rep * D, l % 2 == 1, 20 * seed + l, False)
            norms = [(1 + 0.2 * torch.randn(H, generator=g)).to(BF16).cuda() for _ in range(2)]
            cache = moev.KvCache(s.k.cuda().contiguous(), s.v.cuda().contiguous(), s.ks.cuda(), s.vs.cuda())
            sinks = torch.linspace(-1, 1, self.n_heads).cuda() if l % 2 else None
            self.blocks.append(moev.Block(norms[0], qkv, o, cache, norms[1], layer, window=24 if l % 2 else 0, sinks=sinks))
            self.weights.append((wq, bq, wo, bo))
            self.keep.append(keep)
        self.batch = moev.DraftBatch(torch.tensor(s.cu, dtype=torch.int32).cuda(), torch.tensor(s.ctx, dtype=torch.int32).cuda(), s.table.cuda(),
                                     s.max_drafts, s.max_len, None if s.parent is None else s.parent.cuda())
        self.h = torch.randn(s.T, H, generator=g).to(BF16).cuda()
        self.final = (1 + 0.2 * torch.randn(H, generator=g)).to(BF16).cuda()
        self.rope = s.rope.cuda()

    def outs(self):
        return [self.v.alloc_out(self.T) for _ in self.blocks]

    def step_by_step(self, outs):
        h, y, T = self.h.clone(), None, self.T
        mids = []
        for b, out in zip(self.blocks, outs):
            x, a = torch.empty_like(h), torch.zeros(T, self.n_heads, b.cache.head_dim, dtype=BF16, device="cuda")
            if y is None:
                moev.add_rmsnorm(h, b.attn_norm, {"y": x})
            else:
                moev.add_rmsnorm(y, b.attn_norm, {"y": x, "residual": h}, residual=h)
            qkv = b.qkv(x)
            row, kv = self.n_heads * b.cache.head_dim, b.cache.n_kv_heads * b.cache.head_dim
            q = qkv[:, :row].view(T, self.n_heads, -1)
            moev.cache_append(b.cache, self.batch, qkv[:, row:row + kv].view(T, b.cache.n_kv_heads, -1),
                              qkv[:, row + kv:].view(T, b.cache.n_kv_heads, -1), rope=self.rope, q=q)
            moev.cache_attend(b.cache, self.batch, q, a, window=b.window, sinks=b.sinks)
            mids.append((x.clone(), qkv.clone(), a.clone()))
            moev.add_rmsnorm(b.o(a.view(T, row)), b.ffn_norm, {"y": x, "residual": h}, residual=h)
            mids.append(h.clone())
            self.v.verify(b.layer, x, T, out)
            y = out["y"]
        moev.add_rmsnorm(y, self.final, {"y": x, "residual": h}, residual=h)
        self.v.status_sync()
        return h, x, mids


def setup(tree=True, **kw):
    return R.Setup([20, 0, 131], [4, 3, 5], 32, 2, 4, 64, tree, seed=3, spare=0, **kw)


@pytest.mark.parametrize("base,dims", [("gptoss", dict(H=704, I=320, E=32)), ("qwen", dict(H=1024, I=384, E=32))])
def test_blocks_equal_their_steps(base, dims):
    s = setup()
    a, b = Model(3, s, base, **dims), Model(3, s, base, **dims)
    oa, ob = a.outs(), b.outs()
    h_ref, f_ref, _ = b.step_by_step(ob)
    h, f = a.h.clone(), torch.empty_like(a.h)
    ws = a.v.verify_blocks(a.blocks, a.batch, h, a.n_heads, oa, rope=a.rope, final_norm=a.final, final_out=f)
    a.v.status_sync()
    # the first block's routing and caches come before any MoE output: equal to the bit
    assert torch.equal(oa[0]["topk_ids"], ob[0]["topk_ids"])
    assert torch.equal(a.blocks[0].cache.k.view(torch.uint8), b.blocks[0].cache.k.view(torch.uint8))
    for l in range(3):
        assert torch.equal(oa[l]["topk_ids"], ob[l]["topk_ids"]), f"block {l}"
        assert int(oa[l]["n_active"]) == int(ob[l]["n_active"])
    for got, ref in ((h, h_ref), (f, f_ref)):
        # three MoE outputs, each rounded to bf16 after fp32 additions in another order: a step of bf16 each, and what
        # the later blocks make of it
        assert (got.float() - ref.float()).abs().max() <= 2.0 ** -5 * ref.float().abs().max()
    # again with the same workspace, without the final norm
    h2 = a.h.clone()
    assert a.v.verify_blocks(a.blocks, a.batch, h2, a.n_heads, oa, rope=a.rope, workspace=ws) is ws
    a.v.status_sync()
    assert h2.isfinite().all()
    a.v.close(), b.v.close()


def test_attention_half_of_a_block_against_float64():
    s = setup()
    m = Model(1, s, H=704, I=320, E=32)
    outs = m.outs()
    _, _, mids = m.step_by_step(outs)
    (x, qkv, a), h1 = mids
    wq, bq, wo, _ = m.weights[0]
    _, x_ref = R.rmsnorm(m.h.cpu(), m.blocks[0].attn_norm.cpu(), None, 1e-6)
    assert ((x.cpu().double() - x_ref).abs() <= (2.0 ** -8 * 1.01 + 2.0 ** -17) * x_ref.abs()).all()
    xd = x.cpu().double()
    k_ref = xd @ wq.T + bq.double()
    row = m.n_heads * s.D
    got = qkv.cpu().double()[:, row:]  # k and v as projected (q is rotated in place)
    mass = xd.abs() @ wq.abs().T + bq.double().abs()
    assert ((got - k_ref[:, row:]).abs() <= (2.0 ** -8 * 1.01 * k_ref.abs() + 712 * 2.0 ** -23 * mass)[:, row:]).all()
    c = m.blocks[0].cache
    s.k, s.v, s.ks, s.vs, s.q = c.k.cpu(), c.v.cpu(), c.k_scale.cpu(), c.v_scale.cpu(), qkv[:, :row].cpu().view(s.T, -1, s.D)
    ref, _, pm, ds, floor = s.attend()
    tol = 2.0 ** -8 * 1.01 * ref.abs() + (3 * 2.0 ** -11 + 2.0 ** -14 + 4 * ds)[..., None] * pm + floor
    assert ((a.cpu().double() - ref).abs() <= tol).all()
    ad = a.cpu().double().view(s.T, row)
    o_ref = ad @ wo.T
    h_ref = m.h.cpu().double() + o_ref
    tol = 2.0 ** -8 * 1.01 * (o_ref.abs() + h_ref.abs()) + (row + 8) * 2.0 ** -23 * (ad.abs() @ wo.abs().T) + 2.0 ** -20
    assert ((h1.cpu().double() - h_ref).abs() <= tol).all()
    m.v.close()


def test_blocks_captured_into_a_graph():
    s = setup(tree=False)
    m = Model(2, s, H=704, I=320, E=32)
    outs, h, f = m.outs(), m.h.clone(), torch.empty_like(m.h)
    ws = m.v.verify_blocks(m.blocks, m.batch, h, m.n_heads, outs, rope=m.rope, final_norm=m.final, final_out=f)
    want = f.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.v.verify_blocks(m.blocks, m.batch, h, m.n_heads, outs, rope=m.rope, final_norm=m.final, final_out=f, workspace=ws)
    for _ in range(2):
        h.copy_(m.h)
        f.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert (f.float() - want.float()).abs().max() <= 2.0 ** -5 * want.float().abs().max()
    m.v.status_sync()
    m.v.close()


def test_blocks_refuse_what_does_not_fit():
    s = setup()
    m = Model(1, s, H=704, I=320, E=32)
    outs, b = m.outs(), m.blocks[0]
    call = lambda blocks=m.blocks, h=m.h, heads=m.n_heads, o=outs, **k: m.v.verify_blocks(blocks, m.batch, h, heads, o, **k)  # noqa: E731
    for bad in (lambda: call(h=m.h.float()), lambda: call(h=m.h[:, :512].contiguous()), lambda: call(heads=7), lambda: call(heads=16),
                lambda: call(o=[]), lambda: call(final_norm=m.final), lambda: call(rope=m.rope[:, :32].contiguous()), lambda: call(eps=-1.0),
                lambda: call(h=torch.zeros(s.T + 1, 704, dtype=BF16, device="cuda")),
                lambda: call(blocks=[moev.Block(b.attn_norm, b.o, b.o, b.cache, b.ffn_norm, b.layer)]),
                lambda: call(blocks=[moev.Block(b.attn_norm, b.qkv, b.o, b.cache, b.ffn_norm, b.layer, window=-1)]),
                lambda: call(blocks=[moev.Block(b.attn_norm[:8], b.qkv, b.o, b.cache, b.ffn_norm, b.layer)])):
        with pytest.raises(moev.MoevError):
            bad()
    assert np.isfinite(m.h.float().cpu().numpy()).all()
    m.v.close()


def test_a_refused_call_of_blocks_writes_nothing():
    s = setup()
    m = Model(2, s, H=704, I=320, E=32)
    h, outs, c, b = m.h.clone(), m.outs(), m.blocks[0].cache, m.blocks[1]
    before = [t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale)]
    other = [m.blocks[0], moev.Block(b.attn_norm, b.qkv, b.o, b.cache, b.ffn_norm.cpu(), b.layer)]
    for bad in (lambda: m.v.verify_blocks(m.blocks, m.batch, h, m.n_heads, outs, rope=m.rope, scale=1e9),
                lambda: m.v.verify_blocks(other, m.batch, h, m.n_heads, outs, rope=m.rope)):
        with pytest.raises(moev.MoevError):
            bad()
    torch.cuda.synchronize()
    assert torch.equal(h, m.h)
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip((c.k, c.v, c.k_scale, c.v_scale), before))
    # a workspace with gaps is not written through
    ws = m.v.verify_blocks(m.blocks, m.batch, h, m.n_heads, outs, rope=m.rope)
    gaps = torch.zeros(2 * ws.numel(), dtype=torch.uint8, device="cuda")[::2]
    assert m.v.verify_blocks(m.blocks, m.batch, h, m.n_heads, outs, rope=m.rope, workspace=gaps) is not gaps
    m.v.status_sync()
    assert not gaps.any()
    m.v.close()
