"""Plain float64 forms of the operators around the MoE layer, and the inputs of their tests.

Written from the definitions in include/moev.h with loops over sequences, heads and drafts; used by the
GPU tests and, without a GPU, checked against brute force in test_block_args.py."""
from __future__ import annotations

import math

import torch

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24, torch.float8_e4m3fn: 2.0 ** -4}  # half a step, relative


def rmsnorm(x, w, residual, eps):
    s = x.double() + (0 if residual is None else residual.double())
    return s, s / torch.sqrt(s.square().mean(1, keepdim=True) + eps) * w.double()


def unpack(codes):
    return torch.stack([codes & 15, codes >> 4], 2).flatten(1).long()


def w4_weight(codes, scales, mxfp4, group):
    q = unpack(codes)
    if mxfp4:
        v = torch.tensor(E2M1 + [-e for e in E2M1], dtype=torch.float64, device=q.device)[q]
        s = torch.exp2(scales.double() - 127)
    else:
        v, s = q.double() - 8, scales.double()
    return v * s.repeat_interleave(group, 1)


def decode(codes):
    return codes.view(torch.float8_e4m3fn).double()


def pow2_scale(amax: float) -> float:
    """Smallest power of two s with 448 s >= amax."""
    m, e = math.frexp(amax)
    return math.ldexp(1.0, e - 9 if m <= 0.875 else e - 8)


def ancestors(parent):
    """For each draft of a sequence the list of its ancestors and itself, oldest first."""
    paths = []
    for i, p in enumerate(parent):
        paths.append((paths[p] if 0 <= p < i else []) + [i])
    return paths


def chain(n):
    return [i - 1 for i in range(n)]


def rotate(x, rope_row):
    h = x.shape[-1] // 2
    c, s = rope_row[:h].double(), rope_row[h:].double()
    a, b = x[..., :h].double(), x[..., h:].double()
    return torch.cat([a * c - b * s, b * c + a * s], -1)


class Setup:
    """Sequences with the given context lengths and draft counts over a pool of pages in random order.  What no token has
    been written to holds NaN codes; rows behind the last sequence exist and belong to nobody."""

    def __init__(self, ctx, cnt, page, heads, rep, D, tree=False, seed=0, spare=2, device="cpu", max_len=None, extra_cols=0):
        g = torch.Generator().manual_seed(seed)
        self.ctx, self.cnt, self.page, self.heads, self.rep, self.D = ctx, cnt, page, heads, rep, D
        B = len(ctx)
        self.T = sum(cnt) + spare
        self.cu = [sum(cnt[:b]) for b in range(B + 1)]
        self.max_drafts = max(1, max(cnt))
        self.max_len = max_len or max(max(c + n for c, n in zip(ctx, cnt)), self.max_drafts)
        self.cols = -(-self.max_len // page) + extra_cols
        self.n_pages = B * self.cols + 3
        self.table = torch.randperm(self.n_pages, generator=g)[:B * self.cols].view(B, self.cols).to(torch.int32)
        self.parents = []
        for n in cnt:
            self.parents.append([int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(n)] if tree else chain(n))
        self.tree = tree
        self.parent = torch.tensor([p for ps in self.parents for p in ps] + [-1] * spare, dtype=torch.int32) if tree else None
        val = lambda *s: ((torch.rand(*s, generator=g) - 0.5) * 800).to(torch.float8_e4m3fn)  # noqa: E731
        self.k, self.v = val(self.n_pages, heads, page, D), val(self.n_pages, heads, D, page)
        sc = lambda: torch.exp2(torch.randint(-10, -6, (self.n_pages, heads), generator=g).float())  # noqa: E731
        self.ks, self.vs = sc(), sc()
        self.q = torch.randn(self.T, heads * rep, D, generator=g).to(torch.bfloat16)
        self.nk = (torch.randn(self.T, heads, D, generator=g) * 2).to(torch.bfloat16)
        self.nv = (torch.randn(self.T, heads, D, generator=g) * 2).to(torch.bfloat16)
        angle = torch.arange(self.max_len, dtype=torch.float64)[:, None] * torch.pow(10000.0, -torch.arange(D // 2, dtype=torch.float64) * 2 / D)
        self.rope = torch.cat([angle.cos(), angle.sin()], 1).float()

    def poison(self):
        """NaN codes in every slot of the pool that holds no token of a sequence (its drafts included)."""
        k, v = self.k.view(torch.uint8).clone(), self.v.view(torch.uint8).clone()
        dead = torch.ones(self.n_pages, self.page, dtype=torch.bool)
        for b, (c, n) in enumerate(zip(self.ctx, self.cnt)):
            for j in range(c + n):
                dead[self.table[b, j // self.page].long(), j % self.page] = False
        k[dead[:, None, :, None].expand_as(k)] = 0x7F
        v[dead[:, None, None, :].expand_as(v)] = 0xFF
        self.k, self.v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
        return self

    def position(self, b, i):
        return self.ctx[b] + len(ancestors(self.parents[b])[i]) - 1

    def attend(self, window=0, sinks=None, scale=None):
        """(out, lse, sum of p |v|, bound of the scores' error, floor of the probabilities' error), rows of no sequence as zeros."""
        D, page, rep = self.D, self.page, self.rep
        scale = D ** -0.5 if scale is None else scale
        out = torch.zeros(self.T, self.heads * rep, D, dtype=torch.float64)
        lse, mass = torch.zeros(self.T, self.heads * rep, dtype=torch.float64), torch.zeros_like(out)
        ds, floor = torch.zeros_like(lse), torch.zeros_like(out)
        for b, (c, n) in enumerate(zip(self.ctx, self.cnt)):
            if not n:
                continue
            pages = self.table[b, :-(-(c + n) // page)].long()
            k = (self.k[pages].double() * self.ks[pages].double()[..., None, None]).permute(1, 0, 2, 3).reshape(self.heads, -1, D)
            code = self.v[pages].double().permute(1, 0, 3, 2).reshape(self.heads, -1, D)
            v = (self.v[pages].double() * self.vs[pages].double()[..., None, None]).permute(1, 0, 3, 2).reshape(self.heads, -1, D)
            paths = ancestors(self.parents[b])
            for i, path in enumerate(paths):
                at = c + len(path) - 1
                keys = [j for j in range(max(0, at - window + 1) if window else 0, c)] + [c + j for j in (path[-window:] if window else path)]
                for hq in range(self.heads * rep):
                    kk, vv = k[hq // rep][keys], v[hq // rep][keys]
                    qq = self.q[self.cu[b] + i, hq].double()
                    s = kk @ qq * scale
                    total = torch.logsumexp(s, 0)
                    if sinks is not None:
                        total = torch.logaddexp(total, sinks[hq].double())
                    p = torch.exp(s - total)
                    row = self.cu[b] + i
                    out[row, hq], lse[row, hq], mass[row, hq] = p @ vv, total, p @ vv.abs()
                    # D binary32 additions, each off by at most 2^-23 (the adder may truncate) of the sum of magnitudes
                    # + what is left of q: 2^-18 of its largest element
                    ds[row, hq] = scale * (D * 2.0 ** -23 * (kk.abs() @ qq.abs()).max() + 2.0 ** -18 * qq.abs().max() * kk.abs().sum(1).max())
                    vmax = self.vs[pages][:, hq // rep].double().max()
                    floor[row, hq] = 2.0 ** -19 * p.max() * vmax * code[hq // rep][keys].abs().sum(0)
        return out, lse, mass, ds, floor

    def append(self, rope=True):
        """Expected (q, k values, v values, k_scale, v_scale, bytes that change): k / v values are code-space reals before
        rounding for new tokens (NaN elsewhere)."""
        D, page = self.D, self.page
        q = self.q.double().clone()
        ks, vs = self.ks.double().clone(), self.vs.double().clone()
        new = {"k": torch.full(self.k.shape, math.nan, dtype=torch.float64), "v": torch.full(self.k.shape, math.nan, dtype=torch.float64)}
        kept = {"k": [], "v": []}
        for b, (c, n) in enumerate(zip(self.ctx, self.cnt)):
            for i in range(n):
                row, pos = self.cu[b] + i, self.position(b, i)
                kk, vv = self.nk[row].double(), self.nv[row].double()
                if rope:
                    kk, q[row] = rotate(self.nk[row], self.rope[pos]), rotate(self.q[row], self.rope[pos])
                p = int(self.table[b, (c + i) // page])
                new["k"][p, :, (c + i) % page], new["v"][p, :, (c + i) % page] = kk, vv
            for col in range(c // page, (c + n - 1) // page + 1 if n else c // page):
                p, fill = int(self.table[b, col]), max(0, c - col * page)
                for name, sc in (("k", ks), ("v", vs)):
                    part = new[name][p, :, fill:]
                    for h in range(self.heads):
                        got = part[h][~part[h].isnan()]
                        amax = float(got.abs().max()) if got.numel() else 0.0
                        s = pow2_scale(amax) if amax else 0.0
                        s = max(s, float(sc[p, h])) if fill else (s or 1.0)
                        kept[name].append((p, h, fill, float(sc[p, h]) / s))
                        sc[p, h] = s
        return q, new, kept, ks, vs
