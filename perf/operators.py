"""Operators of a decoder block around the MoE layer, as measured cases.

Four operators of the verification pass over draft tokens, in a plain form (``own = False``:
elementary torch operations in 32 bits, rounded once) and as calls of this framework
(``own = True``):

norm    residual addition + root-mean-square norm, optionally with FP8 1x128 codes and scales
linear  y = x W^T + bias with 4-bit weights: INT4 with bf16 group scales, or MXFP4
append  rotary positions, and keys / values written to a paged 8-bit cache with one power-of-two
        scale per page and head
attend  attention of the drafts over that cache: the prefix (optionally a window of it) and each
        draft's ancestors in the tree, optional sink logits
"""
import math

import torch

own = False

BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
TYPES = {"bf16": BF16, "fp32": F32}


# ------------------------------------------------------------------ cases

def listed():
    return [
        # the hidden states of one draft chain between two layers
        dict(name="norm_drafts", op="norm", n=4, H=4096, act="bf16", residual=True, quant=0, pad=0),
        # a full draft tree in front of FP8 projections: both forms of the output
        dict(name="norm_tree_fp8", op="norm", n=64, H=7168, act="bf16", residual=True, quant=1, pad=0),
        # a prompt's hidden states, rows wider than the norm (a slice of a fused buffer)
        dict(name="norm_prompt", op="norm", n=8192, H=7168, act="bf16", residual=True, quant=2, pad=64),
        # output projection for a single token
        dict(name="linear_token", op="linear", n=1, N=4096, K=8192, fmt="int4", group=128, out="bf16", bias=False),
        # fused query / key / value projection of a small draft tree, a width that is no multiple of 128
        dict(name="linear_drafts", op="linear", n=8, N=5120, K=2880, fmt="mxfp4", group=32, out="bf16", bias=True),
        # logits of a draft tree over a vocabulary of odd size
        dict(name="linear_vocab", op="linear", n=16, N=100003, K=7168, fmt="int4", group=64, out="fp32", bias=False),
        # a draft tree written behind a context that ends inside a page
        dict(name="append_tree", op="append", B=1, n=64, ragged=False, ctx=4099, kv=8, rep=8, D=64, page=16, tree=True, rope=True),
        # chunks of several prompts
        dict(name="append_prompts", op="append", B=8, n=1024, ragged=True, ctx=5000, kv=8, rep=8, D=128, page=64, tree=False, rope=True),
        # one token of one sequence: ordinary decoding
        dict(name="attend_token", op="attend", B=1, n=1, ragged=False, ctx=4095, kv=4, rep=16, D=128, page=64, tree=False, window=0, sinks=False),
        # a full draft tree over a long context
        dict(name="attend_tree", op="attend", B=1, n=64, ragged=False, ctx=16001, kv=4, rep=16, D=128, page=128, tree=True, window=0, sinks=False),
        # a serving batch of ragged contexts, a few drafts each
        dict(name="attend_batch", op="attend", B=32, n=4, ragged=True, ctx=24000, kv=8, rep=8, D=128, page=64, tree=True, window=0, sinks=False),
        # a sliding-window layer with sink logits
        dict(name="attend_window", op="attend", B=16, n=8, ragged=True, ctx=6000, kv=8, rep=8, D=64, page=16, tree=True, window=128, sinks=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm", "linear", "append", "attend"))
    if op == "norm":
        return dict(op=op, n=_log(rng, 1, 6000), H=rng.choice((256, 704, 1000, 2880, 4096, 7168)), act=rng.choice(("bf16", "bf16", "fp32")),
                    residual=rng.random() < 0.75, quant=rng.choice((0, 1, 2)), pad=rng.choice((0, 0, 32)))
    if op == "linear":
        fmt = rng.choice(("int4", "int4", "mxfp4"))
        group = 32 if fmt == "mxfp4" else rng.choice((32, 64, 128))
        return dict(op=op, n=_log(rng, 1, 16), N=_log(rng, 100, 60000), K=group * _log(rng, 2, 7168 // group), fmt=fmt, group=group,
                    out=rng.choice(("bf16", "fp32")), bias=rng.random() < 0.5)
    D = rng.choice((64, 128))
    kv = rng.choice((1, 2, 4, 8))
    rep = rng.choice((1, 3, 4, 8, 16) if kv <= 4 else (1, 4, 8))
    if op == "append":
        B = _log(rng, 1, 16)
        tree = rng.random() < 0.5
        return dict(op=op, B=B, n=_log(rng, 1, 64 if tree else 4000 // B), ragged=rng.random() < 0.7, ctx=_log(rng, 1, 5000), kv=kv, rep=rep, D=D,
                    page=rng.choice((16, 32, 64, 128)), tree=tree, rope=rng.random() < 0.8)
    B = _log(rng, 1, 32)
    return dict(op=op, B=B, n=_log(rng, 1, 64 if B * kv * rep <= 64 else 4), ragged=rng.random() < 0.7, ctx=_log(rng, 1, 16000 if B < 16 else 8000), kv=kv, rep=rep, D=D,
                page=rng.choice((16, 32, 64, 128)), tree=rng.random() < 0.6, window=rng.choice((0, 0, 128, 1000)), sinks=rng.random() < 0.3)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * (int(seed) + 1))


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", dtype=F32, generator=g)


def _drafts(case, g):
    """Sequences of the call: offsets, context lengths, page table, parents; lengths are host numbers too."""
    B, n, page = case["B"], case["n"], case["page"]
    if case["ragged"]:
        u = torch.rand(2, B, device="cuda", generator=g).cpu()
        cnt = (u[0] * (n + 1)).long().clamp(max=n)  # a sequence may bring no draft at all
        ctx = (u[1] * (case["ctx"] + 1)).long().clamp(max=case["ctx"])
        cnt[0], ctx[-1] = n, case["ctx"]
    else:
        cnt, ctx = torch.full((B,), n), torch.full((B,), case["ctx"])
    cu = torch.cat([torch.zeros(1, dtype=torch.long), cnt.cumsum(0)])
    T = B * n + (3 if case["ragged"] else 0)  # a padded batch: rows behind the last sequence belong to nobody
    max_len = case["ctx"] + n
    cols = -(-max_len // page)
    n_pages = B * cols + 1
    table = torch.randperm(n_pages, device="cuda", generator=g)[:B * cols].view(B, cols)
    parent = None
    if case["tree"]:
        local = torch.cat([torch.arange(int(c)) for c in cnt] + [torch.zeros(T - int(cu[-1]), dtype=torch.long)]).cuda()
        r = torch.rand(T, device="cuda", generator=g)
        parent = ((r * (local + 1)).long() - 1).to(torch.int32)  # -1: the draft hangs on the context
    return dict(T=T, cnt=cnt, ctx_h=ctx, cu=cu.to(torch.int32).cuda(), ctx=ctx.to(torch.int32).cuda(), table=table.to(torch.int32),
                parent=parent, n_pages=n_pages, max_len=max_len, cols=cols)


def prepare(case, seed):
    g, op, s = _gen(seed), case["op"], {}
    s["case"] = case
    if op == "norm":
        n, H, t = case["n"], case["H"], TYPES[case["act"]]
        wide = H + case["pad"]
        s["x"] = (_randn(g, n, wide) * 0.7).to(t)[:, :H]
        s["res"] = (_randn(g, n, wide) * 2).to(t)[:, :H] if case["residual"] else None
        s["w"] = (1 + 0.2 * _randn(g, H)).to(t)
        s["out"] = {"y": torch.empty(n, H, device="cuda", dtype=t)}
        if case["residual"]:
            s["out"]["residual"] = torch.empty(n, H, device="cuda", dtype=t)
        if case["quant"]:
            s["out"]["codes"] = torch.empty(n, H, device="cuda", dtype=F8)
            s["out"]["scales"] = torch.empty(n, -(-H // 128), device="cuda", dtype=F32)
    elif op == "linear":
        n, N, K, group = case["n"], case["N"], case["K"], case["group"]
        s["x"] = _randn(g, n, K).to(BF16)
        s["codes"] = torch.randint(0, 256, (N, K // 2), device="cuda", dtype=torch.uint8, generator=g)
        if case["fmt"] == "int4":
            s["scales"] = (torch.rand(N, K // group, device="cuda", generator=g) * 0.006 + 0.002).to(BF16)
        else:
            s["scales"] = torch.randint(115, 122, (N, K // 32), device="cuda", dtype=torch.uint8, generator=g)
        s["bias"] = _randn(g, N) * 0.1 if case["bias"] else None
        s["y"] = torch.empty(n, N, device="cuda", dtype=TYPES[case["out"]])
        if own:
            import paper_2607_12696_b200 as moev
            s["lin"] = moev.W4Linear(s["codes"], s["scales"], moev.W_INT4 if case["fmt"] == "int4" else moev.W_MXFP4, group, s["bias"])
    else:
        d = _drafts(case, g)
        s.update(d)
        kv, D, page, hq = case["kv"], case["D"], case["page"], case["kv"] * case["rep"]
        codes = lambda *shape: (torch.rand(*shape, device="cuda", dtype=BF16, generator=g).sub_(0.5) * 600).to(F8)  # noqa: E731
        s["k"], s["v"] = codes(d["n_pages"], kv, page, D), codes(d["n_pages"], kv, D, page)
        s["ks"] = torch.exp2(torch.randint(-9, -5, (d["n_pages"], kv), device="cuda", generator=g).float())
        s["vs"] = torch.exp2(torch.randint(-9, -5, (d["n_pages"], kv), device="cuda", generator=g).float())
        s["q"] = _randn(g, d["T"], hq, D).to(BF16)
        if op == "append":
            qkv = torch.cat([s["q"].reshape(d["T"], hq * D), (_randn(g, d["T"], 2 * kv * D) * 1.5).to(BF16)], 1)  # one projection's output
            s["q"] = qkv[:, :hq * D].view(d["T"], hq, D)
            s["nk"] = qkv[:, hq * D:(hq + kv) * D].view(d["T"], kv, D)
            s["nv"] = qkv[:, (hq + kv) * D:].view(d["T"], kv, D)
            s["rope"] = None
            if case["rope"]:
                angle = torch.arange(d["max_len"], device="cuda", dtype=torch.float64)[:, None] * torch.pow(
                    150000.0, -torch.arange(D // 2, device="cuda", dtype=torch.float64) * 2 / D)
                s["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float()
            s["q_out"] = torch.zeros(d["T"], hq, D, device="cuda", dtype=BF16)
        else:
            # slots that no token has been written to hold whatever was there: here, NaN
            end = (d["ctx_h"] + d["cnt"]).cuda()[:, None]
            slot = torch.arange(d["cols"] * page, device="cuda")[None]
            dead = (slot >= end).view(-1, page)
            pages = d["table"].long().view(-1)
            km, vm = s["k"].view(torch.uint8), s["v"].view(torch.uint8)
            km[pages] = torch.where(dead[:, None, :, None], 0x7F, km[pages])
            vm[pages] = torch.where(dead[:, None, None, :], 0x7F, vm[pages])
            s["sinks"] = _randn(g, hq) if case["sinks"] else None
            s["out"] = torch.zeros(d["T"], hq, D, device="cuda", dtype=BF16)
            s["lse"] = torch.zeros(d["T"], hq, device="cuda", dtype=F32)
        if own:
            import paper_2607_12696_b200 as moev
            s["cache"] = moev.KvCache(s["k"], s["v"], s["ks"], s["vs"])
            s["batch"] = moev.DraftBatch(s["cu"], s["ctx"], s["table"], case["n"], d["max_len"], s["parent"])
            if op == "attend":
                s["work"] = moev.cache_attend_workspace(s["cache"], s["batch"], hq)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        import paper_2607_12696_b200 as moev
        if op == "norm":
            moev.add_rmsnorm(s["x"], s["w"], s["out"], residual=s["res"], eps=1e-6, act_quant=case["quant"])
            return s["out"]
        if op == "linear":
            return s["lin"](s["x"], s["y"])
        if op == "append":
            moev.cache_append(s["cache"], s["batch"], s["nk"], s["nv"], rope=s["rope"], q=s["q"], q_out=s["q_out"])
            return _append_result(s)
        moev.cache_attend(s["cache"], s["batch"], s["q"], s["out"], lse=s["lse"], window=case["window"], sinks=s["sinks"], workspace=s["work"])
        return {"out": s["out"], "lse": s["lse"]}
    return {"norm": _norm, "linear": _linear, "append": _append, "attend": _attend}[op](s)


def _append_result(s):
    return {"q": s["q_out"], "k": s["k"], "v": s["v"], "k_scale": s["ks"], "v_scale": s["vs"]}


def _over_448(x):
    return x / torch.full_like(x, 448.0)  # a true division: by a number, it would be a product with the rounded reciprocal


def _pow2_at_least(x):
    m, e = torch.frexp(x)
    return torch.ldexp(torch.ones_like(x), torch.where(m == 0.5, e - 1, e))


def _norm(s):
    case, x = s["case"], s["x"]
    t, n, H = x.dtype, case["n"], case["H"]
    r = x.float() if s["res"] is None else x.float() + s["res"].float()
    y = r * torch.rsqrt(r.square().mean(1, keepdim=True) + 1e-6) * s["w"].float()
    out = {"y": y.to(t)}
    if s["res"] is not None:
        out["residual"] = r.to(t)
    if case["quant"]:
        blocks = -(-H // 128)
        yp = torch.zeros(n, blocks * 128, device=y.device)
        yp[:, :H] = y
        yp = yp.view(n, blocks, 128)
        scale = _over_448(yp.abs().amax(2))
        if case["quant"] == 2:
            scale = _pow2_at_least(scale)
        scale = torch.where(scale == 0, 1.0, scale)
        out["codes"] = (yp / scale[:, :, None]).clamp(-448, 448).view(n, -1)[:, :H].to(F8)
        out["scales"] = scale
    return out


def _nibbles(codes):
    return torch.stack([codes & 15, codes >> 4], 2).flatten(1).long()


def _linear(s):
    case = s["case"]
    q = _nibbles(s["codes"])
    if case["fmt"] == "int4":
        w, scale = (q - 8).float(), s["scales"].float()
    else:
        mag = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=q.device)
        w, scale = mag[q], torch.exp2(s["scales"].float() - 127)
    w = (w.view(case["N"], -1, case["group"]) * scale[:, :, None]).view(case["N"], -1)
    y = s["x"].float() @ w.T
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["y"].dtype)


def _rows(s):
    """For every token: its sequence and its place in it (tokens behind the last sequence excluded)."""
    cu, B = s["cu"].long(), s["case"]["B"]
    tok = torch.arange(s["T"], device=cu.device)
    seq = torch.bucketize(tok, cu[1:], right=True)
    live = seq < B
    tok, seq = tok[live], seq[live]
    return tok, seq, tok - cu[seq]


def _seen(s):
    """[B, n, n]: draft i sees draft j (itself and its ancestors)."""
    case = s["case"]
    B, n = case["B"], case["n"]
    if s["parent"] is None:
        return torch.ones(n, n, device=s["cu"].device).tril().expand(B, n, n) > 0
    tok, seq, i = _rows(s)
    par = s["parent"][tok].long()
    has = par >= 0
    step = torch.eye(n, device=tok.device, dtype=torch.float64).repeat(B, 1, 1)
    step[seq[has], i[has], par[has]] = 1
    return torch.linalg.matrix_power(step, max(1, n - 1)) > 0


def _append(s):
    case = s["case"]
    D, page = case["D"], case["page"]
    tok, seq, i = _rows(s)
    seen = _seen(s)
    pos = s["ctx"].long()[seq] + seen.sum(2)[seq, i] - 1
    k, v, q = s["nk"][tok].float(), s["nv"][tok].float(), s["q"][tok].float()
    if s["rope"] is not None:
        cos, sin = (a[:, None, :] for a in s["rope"][pos].split(D // 2, 1))
        turn = lambda a: torch.cat([a[..., :D // 2] * cos - a[..., D // 2:] * sin, a[..., D // 2:] * cos + a[..., :D // 2] * sin], 2)  # noqa: E731
        k, q = turn(k), turn(q)
    s["q_out"][tok] = q.to(BF16)
    slot = s["ctx"].long()[seq] + i
    where, off = s["table"].long()[seq, slot // page], slot % page
    first = s["ctx"].long()  # a page that is part full holds the tokens in front of the first new one
    partial = (first % page > 0) & (s["cu"][1:] > s["cu"][:-1])
    col = (first // page).clamp(max=s["cols"] - 1)
    kept = s["table"].long()[torch.arange(case["B"], device=tok.device), col][partial]
    old = torch.arange(page, device=tok.device)[None] < (first % page)[partial][:, None]  # [parts, page]
    for new, codes, scale, tr in ((k, s["k"], s["ks"], False), (v, s["v"], s["vs"], True)):
        amax = torch.zeros_like(scale).index_reduce_(0, where, new.abs().amax(2), "amax")
        want = _pow2_at_least(_over_448(amax))
        want = torch.where(amax == 0, 1.0, want)
        touched = torch.zeros(scale.shape[0], dtype=torch.bool, device=tok.device).index_fill_(0, where, True)[:, None]
        was = scale.clone()
        keep = torch.zeros(scale.shape[0], dtype=torch.bool, device=tok.device).index_fill_(0, kept, True)[:, None]
        now = torch.where(touched, torch.where(keep, torch.maximum(torch.where(amax == 0, 0.0, want), was), want), was)
        ratio = (was / now)[kept]  # [parts, heads]
        view = codes.transpose(2, 3) if tr else codes
        part = view[kept].float()
        part = torch.where(old[:, None, :, None], part * ratio[:, :, None, None], part)  # the other slots as they are
        view.view(torch.uint8)[kept] = part.to(F8).view(torch.uint8)
        enc = (new / now[where][:, :, None]).clamp(-448, 448).to(F8).view(torch.uint8)
        view.view(torch.uint8)[where, :, off] = enc
        scale.copy_(now)
    return _append_result(s)


def _attend(s):
    case = s["case"]
    B, n, kv, rep, D, page = (case[x] for x in ("B", "n", "kv", "rep", "D", "page"))
    tok, seq, i = _rows(s)
    S = s["cols"] * page
    pages = s["table"].long()
    at = torch.arange(S, device=tok.device)
    ctx = s["ctx"].long()
    seen = _seen(s)  # [B, n, n]
    depth = seen.sum(2) - 1
    local = at[None] - ctx[:, None]  # [B, S]: the draft in a slot, negative for the context
    count = (s["cu"][1:] - s["cu"][:-1]).long()
    of = local.clamp(0, n - 1)
    kpos = torch.where(local < 0, at[None], ctx[:, None] + depth.gather(1, of))
    qpos = ctx[:, None] + depth  # [B, n]
    ok = torch.where((local < 0)[:, None], True, seen.gather(2, of[:, None].expand(B, n, S)) & (local < count[:, None])[:, None])
    if case["window"]:
        ok = ok & (kpos[:, None] > qpos[:, :, None] - case["window"])
    written = (local < count[:, None])[:, None, :, None]
    load = lambda codes, scale: torch.where(written, (codes[pages].float() * scale[pages][..., None, None]).transpose(1, 2).reshape(B, kv, S, D), 0.0)  # noqa: E731
    k, v = load(s["k"], s["ks"]), load(s["v"].transpose(2, 3), s["vs"])
    q = torch.zeros(B, n, kv * rep, D, device=tok.device)
    q[seq, i] = s["q"][tok].float()
    q = q.view(B, n, kv, rep, D).permute(0, 2, 1, 3, 4).reshape(B, kv, n * rep, D)
    score = (q @ k.transpose(2, 3)).view(B, kv, n, rep, S) / math.sqrt(D)
    score = score.masked_fill(~ok[:, None, :, None, :], -math.inf)
    top = score.amax(4, keepdim=True)
    sink = None
    if s["sinks"] is not None:
        sink = s["sinks"].view(1, kv, 1, rep, 1)
        top = torch.maximum(top, sink)
    p = torch.exp(score - top)
    total = p.sum(4, keepdim=True)
    if sink is not None:
        total = total + torch.exp(sink - top)
    o = (p.view(B, kv, n * rep, S) @ v).view(B, kv, n, rep, D) / total
    lse = (torch.log(total) + top)[..., 0]
    out, l_out = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    out[tok] = o.permute(0, 2, 1, 3, 4).reshape(B, n, kv * rep, D)[seq, i].to(BF16)
    l_out[tok] = lse.permute(0, 2, 1, 3).reshape(B, n, kv * rep)[seq, i]
    return {"out": out, "lse": l_out}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "norm":
        n, H, b = case["n"], case["H"], 2 if case["act"] == "bf16" else 4
        per = b * (2 + 2 * case["residual"]) + (1 + 4 / 128 if case["quant"] else 0)
        return {"bytes": n * H * per + H * b, "flops": n * H * 5.0}
    if op == "linear":
        n, N, K = case["n"], case["N"], case["K"]
        scales = N * (K // case["group"]) * (2 if case["fmt"] == "int4" else 1)
        return {"bytes": N * K / 2 + scales + n * K * 2 + n * N * (2 if case["out"] == "bf16" else 4) + (4 * N if case["bias"] else 0), "flops": 2.0 * n * N * K}
    kv, rep, D, B = case["kv"], case["rep"], case["D"], case["B"]
    tokens = B * case["n"] * (0.55 if case["ragged"] else 1.0)
    if op == "append":
        return {"bytes": tokens * D * (4 * kv * rep + 6 * kv), "flops": tokens * D * (6 * kv * rep + 10 * kv)}
    ctx = case["ctx"] * (0.5 if case["ragged"] else 1.0)
    if case["window"]:
        ctx = min(ctx, case["window"])
    seen = ctx + (case["n"] + 1) / 2
    return {"bytes": B * (ctx + case["n"]) * kv * D * 2 + tokens * kv * rep * (4 * D + 4), "flops": tokens * kv * rep * seen * D * 4.0}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _norm64, "linear": _linear64, "append": _append64, "attend": _attend64}[case["op"]](s)


def _grid64(amax):
    m, e = torch.frexp(amax)  # 448 = 0.875 * 2^9: the smallest power of two that brings amax to 448 or less
    return torch.ldexp(torch.ones_like(amax), torch.where(m <= 0.875, e - 9, e - 8))


def _norm64(s):
    case = s["case"]
    h = s["x"].double()
    out = {}
    if s["res"] is not None:
        h = h + s["res"].double()
        out["residual"] = h
    y = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["H"] + 1e-6) * s["w"].double()
    out["y"] = y
    if case["quant"]:
        codes, scales = torch.empty_like(y), []
        for a in range(0, case["H"], 128):
            b = y[:, a:a + 128]
            top = b.abs().max(1, keepdim=True).values
            sc = top / 448 if case["quant"] == 1 else _grid64(top)
            codes[:, a:a + 128] = b / sc
            scales.append(sc)
        out["codes"], out["scales"] = codes, torch.cat(scales, 1)
    return out


def _linear64(s):
    case = s["case"]
    N, K, group = case["N"], case["K"], case["group"]
    x, parts = s["x"].double(), []
    for a in range(0, N, 8192):
        c = s["codes"][a:a + 8192].int()
        w = torch.empty(c.shape[0], K, device=c.device, dtype=torch.float64)
        for half in range(2):
            q = (c >> (4 * half)) & 15
            if case["fmt"] == "int4":
                w[:, half::2] = q.double() - 8
            else:
                e, m = (q >> 1) & 3, (q & 1).double()
                mag = torch.where(e == 0, m / 2, (1 + m / 2) * 2.0 ** (e.double() - 1))
                w[:, half::2] = torch.where(q >= 8, -mag, mag)
        sc = s["scales"][a:a + 8192]
        sc = sc.double() if case["fmt"] == "int4" else 2.0 ** (sc.double() - 127)
        parts.append(x @ (w * sc.repeat_interleave(group, 1)).T)
    y = torch.cat(parts, 1)
    return y if s["bias"] is None else y + s["bias"].double()


def _paths(s, b):
    """Ancestor lists of one sequence's drafts, by following the parents."""
    lo, cnt = int(s["cu"][b]), int(s["cnt"][b])
    if s["parent"] is None:
        return None
    par, paths = s["parent"][lo:lo + cnt].tolist(), []
    for i in range(cnt):
        paths.append([i] if par[i] < 0 else paths[par[i]] + [i])
    return paths


def _append64(s):
    case = s["case"]
    D, page, kv = case["D"], case["page"], case["kv"]
    q_out = s["q_out"].double()
    k, v, ks, vs = s["k"].double(), s["v"].double(), s["ks"].double(), s["vs"].double()
    for b in range(case["B"]):
        lo, cnt, ctx = int(s["cu"][b]), int(s["cnt"][b]), int(s["ctx_h"][b])
        if not cnt:
            continue
        paths = _paths(s, b)
        pos = torch.arange(cnt) if paths is None else torch.tensor([len(p) - 1 for p in paths])
        pos = (pos + ctx).to(k.device)
        rows = slice(lo, lo + cnt)
        nq, nk, nv = s["q"][rows].double(), s["nk"][rows].double(), s["nv"][rows].double()
        if s["rope"] is not None:
            z = torch.complex(s["rope"][pos, :D // 2].double(), s["rope"][pos, D // 2:].double())[:, None]
            spin = lambda a: (lambda c: torch.cat([c.real, c.imag], 2))(torch.complex(a[..., :D // 2], a[..., D // 2:]) * z)  # noqa: E731
            nq, nk = spin(nq), spin(nk)
        q_out[rows] = nq
        for c in range(ctx // page, (ctx + cnt - 1) // page + 1):
            p = int(s["table"][b, c])
            first, last = max(ctx, c * page), min(ctx + cnt, (c + 1) * page)
            fill = first - c * page
            for new, codes, scale in ((nk, k[p], ks), (nv, v[p].transpose(1, 2), vs)):
                part = new[first - ctx:last - ctx].transpose(0, 1)  # [kv, tokens, D]
                amax = part.abs().amax((1, 2))
                want = torch.where(amax > 0, _grid64(amax), 0.0)
                sc = torch.maximum(want, scale[p]) if fill else torch.where(want > 0, want, 1.0)
                codes[:, :fill] *= (scale[p] / sc)[:, None, None]
                codes[:, fill:fill + last - first] = part / sc[:, None, None]
                scale[p] = sc
    return {"q": q_out, "k": k, "v": v, "k_scale": ks, "v_scale": vs}


def _attend64(s):
    case = s["case"]
    D, page, kv, rep = case["D"], case["page"], case["kv"], case["rep"]
    out, lse = s["out"].double(), s["lse"].double()
    for b in range(case["B"]):
        lo, cnt, ctx = int(s["cu"][b]), int(s["cnt"][b]), int(s["ctx_h"][b])
        if not cnt:
            continue
        paths = _paths(s, b) or [list(range(i + 1)) for i in range(cnt)]
        end = ctx + cnt
        pages = s["table"][b, :-(-end // page)].long()
        k = (s["k"][pages].double() * s["ks"][pages].double()[..., None, None]).permute(1, 0, 2, 3).reshape(kv, -1, D)[:, :end]
        v = (s["v"][pages].double() * s["vs"][pages].double()[..., None, None]).permute(1, 0, 3, 2).reshape(kv, -1, D)[:, :end]
        for h in range(kv):
            q = s["q"][lo:lo + cnt, h * rep:(h + 1) * rep].double()
            logit = torch.einsum("nrd,sd->nrs", q, k[h]) * D ** -0.5
            hide = torch.ones(cnt, end, dtype=torch.bool)
            for i, path in enumerate(paths):
                at = ctx + len(path) - 1
                start = max(0, at - case["window"] + 1) if case["window"] else 0
                hide[i, start:ctx] = False
                keep = path if not case["window"] else path[-case["window"]:]
                hide[i, [ctx + j for j in keep]] = False
            logit = logit.masked_fill(hide.to(logit.device)[:, None], -math.inf)
            total = torch.logsumexp(logit, 2)
            if s["sinks"] is not None:
                total = torch.logaddexp(total, s["sinks"][h * rep:(h + 1) * rep].double()[None])
            out[lo:lo + cnt, h * rep:(h + 1) * rep] = torch.einsum("nrs,sd->nrd", torch.exp(logit - total[..., None]), v[h])
            lse[lo:lo + cnt, h * rep:(h + 1) * rep] = total
    return {"out": out, "lse": lse}
