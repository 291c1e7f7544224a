"""moev_verify_blocks itself, beyond its first caches: a block's call against the steps called one by one (which
test_gpu_blocks.py compares with float64), to the bit, and every block's caches in a call of three."""
import pytest
import torch

from test_gpu_blocks import Model, setup

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("l", [0, 1])
def test_one_block_is_its_steps_to_the_bit(l, tree):
    """Both kinds of block (formats, window, sinks): cache, routing, and the stream behind it, which is the steps' stream in
    front of the MoE layer plus the MoE output that the call returned, rounded once."""
    s = setup(tree)
    a, b = Model(2, s, H=704, I=320, E=32), Model(2, s, H=704, I=320, E=32)
    a.blocks, b.blocks = a.blocks[l:l + 1], b.blocks[l:l + 1]
    oa, ob = a.outs(), b.outs()
    _, _, mids = b.step_by_step(ob)
    h = a.h.clone()
    a.v.verify_blocks(a.blocks, a.batch, h, a.n_heads, oa, rope=a.rope)
    a.v.status_sync()
    x, y = a.blocks[0].cache, b.blocks[0].cache
    for name in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(x, name).view(torch.uint8), getattr(y, name).view(torch.uint8)), name
    assert torch.equal(oa[0]["topk_ids"], ob[0]["topk_ids"]) and torch.equal(oa[0]["topk_w"], ob[0]["topk_w"])
    assert torch.equal(h, (mids[1].float() + oa[0]["y"].float()).to(BF16))
    assert not torch.equal(mids[1], a.h)
    a.v.close(), b.v.close()


@pytest.mark.parametrize("base,dims", [("gptoss", dict(H=704, I=320, E=32)), ("qwen", dict(H=1024, I=384, E=32))])
def test_every_block_uses_its_own_weights_and_cache(base, dims):
    """Three blocks of different formats, windows and sinks in one call: caches of the first to the bit, of the others within
    what a step of bf16 in the stream makes of a projection."""
    s = setup()
    a, b = Model(3, s, base, **dims), Model(3, s, base, **dims)
    oa, ob = a.outs(), b.outs()
    _, _, mids = b.step_by_step(ob)
    a.v.verify_blocks(a.blocks, a.batch, a.h.clone(), a.n_heads, oa, rope=a.rope)
    a.v.status_sync()
    row, kv = a.n_heads * s.D, s.heads * s.D
    for l in range(3):
        ca, cb = a.blocks[l].cache, b.blocks[l].cache
        if l == 0:
            for x, y in ((ca.k, cb.k), (ca.v, cb.v), (ca.k_scale, cb.k_scale), (ca.v_scale, cb.v_scale)):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
            continue
        x, qkv, _ = mids[2 * l]
        wq = a.weights[l][0].abs().cuda()
        # every element of x may be off by two steps: their products' magnitudes, added like a root over the columns
        bound = 4 * 2.0 ** -8 * (x.double().square() @ wq.square().T).sqrt()
        for at, pa, pb, sa, sb in ((row, ca.k, cb.k, ca.k_scale, cb.k_scale), (row + kv, ca.v.transpose(2, 3), cb.v.transpose(2, 3), ca.v_scale, cb.v_scale)):
            va, vb = (p.float().double() * t.double()[:, :, None, None] for p, t in ((pa, sa), (pb, sb)))
            for seq, (c, n) in enumerate(zip(s.ctx, s.cnt)):
                for i in range(n):
                    p, off = int(s.table[seq, (c + i) // s.page]), (c + i) % s.page
                    got, want = va[p, :, off], vb[p, :, off]
                    lim = bound[s.cu[seq] + i, at:at + kv].view(s.heads, s.D).amax(1, keepdim=True) * 1.5 + 2.0 ** -3 * want.abs() + \
                        2.0 ** -9 * torch.maximum(sa[p], sb[p]).double()[:, None]
                    assert ((got - want).abs() <= lim).all()
                    assert (lim < 0.7 * want.abs().amax(1, keepdim=True)).any()
    a.v.close(), b.v.close()
