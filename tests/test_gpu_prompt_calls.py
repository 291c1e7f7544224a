"""Calls of the operators in front of and behind a verification pass that programs make beside the plain ones: none of the keys, one row of a
larger tensor, several streams, threads and replayed graphs at once, the same tensors twice."""
import threading

import pytest
import torch

import paper_2607_12696_b200 as moev
import prompt_ref as R

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def t32(v):
    return torch.tensor(v, dtype=I32, device="cuda")


@pytest.mark.parametrize("D", [64, 128])
def test_prompt_without_any_key_or_sequence(D):
    q, none = torch.randn(7, 4, D, device="cuda").to(BF16), torch.empty(0, 2, D, dtype=BF16, device="cuda")
    out, lse = torch.full_like(q, 7), torch.full((7, 4), 7.0, device="cuda")
    moev.prompt_attend(moev.PromptBatch(t32([0, 2, 5]), 3, cu_k=t32([0, 0, 0])), q, none, none, out, lse)
    assert (out[:5] == 0).all() and (lse[:5] == -torch.inf).all() and (out[5:] == 7).all() and (lse[5:] == 7).all()
    out.fill_(7)
    moev.prompt_attend(moev.PromptBatch(t32([0]), 3), q, q[:, :2], q[:, 2:], out)
    assert (out == 7).all()
    empty = q[:0]
    assert moev.prompt_attend(moev.PromptBatch(t32([0, 0]), 1), empty, empty[:, :2], empty[:, :2]).shape == (0, 4, D)


@pytest.mark.parametrize("D", [64, 128])
def test_one_row_of_larger_tensors(D):
    """Strides of a single row are not looked at, whatever they are."""
    g = torch.Generator().manual_seed(D)
    wide = torch.randn(5, 12 * D + 3, generator=g).to(BF16).cuda()  # rows on no 16-byte boundary but the first
    q, k, v = wide[:1, :8 * D].view(1, 8, D), wide[:1, 8 * D:10 * D].view(1, 2, D), wide[:1, 10 * D:12 * D].view(1, 2, D)
    out = moev.prompt_attend(moev.PromptBatch(t32([0, 1]), 1), q, k, v)
    assert torch.equal(out, v.repeat_interleave(4, 1))
    w, scales = torch.randint(-127, 128, (40, 64), generator=g, dtype=torch.int8).cuda(), torch.rand(40, generator=g).cuda()
    lin, x = moev.W8Linear(w, scales), wide[:1, :64]
    want, tol = R.linear(*R.quantize(x), w, scales, None, F32)
    y = torch.full((3, 43), 7.0, device="cuda")
    lin(x, y[1:2, :40])
    assert ((y[1:2, :40].double() - want).abs() <= tol).all() and (y[0] == 7).all() and (y[2] == 7).all() and (y[1, 40:] == 7).all()
    logits = wide[2:3, 5:1000 if D == 128 else 700].float()
    big = torch.cat([logits, logits], 1)[:, 1:]
    lse = torch.empty(1, device="cuda")
    moev.token_logprobs(big, None, {"lse": lse})
    assert abs(float(lse) - float(torch.logsumexp(big.double(), 1))) < 1e-5


def programs():
    """Every operator and each of its forms as a closure that returns its outputs, with inputs and outputs of its own."""
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    res = []

    def attend(n_q, n_k, kv, rep, D, most, empty):
        cu, cu_k = [0], [0]
        for a, b in zip(n_q + [0] * empty, n_k + [0] * empty):
            cu.append(cu[-1] + a)
            cu_k.append(cu_k[-1] + b)
        q, k, v = rnd(cu[-1], kv * rep, D).to(BF16), rnd(cu_k[-1], kv, D).to(BF16), rnd(cu_k[-1], kv, D).to(BF16)
        batch = moev.PromptBatch(t32(cu), most, cu_k=t32(cu_k))

        def call():
            lse = torch.empty(cu[-1], kv * rep, device="cuda")
            return moev.prompt_attend(batch, q, k, v, torch.empty_like(q), lse), lse
        res.append(call)

    attend([300, 40], [600, 40], 2, 4, 128, 300, 0)      # one tile of rows
    attend([20], [4000], 2, 4, 64, 20, 0)                # keys shared by a cluster
    attend([1500, 700], [1500, 700], 2, 4, 128, 1500, 100)  # two tiles of rows
    for n, N, K in ((1, 4096, 2048), (2, 300, 4096), (50, 2000, 2880), (100, 700, 1024), (2000, 3000, 1024)):
        lin, x = moev.W8Linear(*moev.quantize_rows(rnd(N, K))), rnd(n, K).to(BF16)
        res.append(lambda lin=lin, x=x, n=n: (lin(x, torch.empty(n, lin.N, device="cuda")),))
        res.append(lambda lin=lin, x=x: (lin(moev.quantize_rows(x)),))
    for n, V, dtype in ((1, 100003, F32), (64, 30011, BF16), (700, 5000, F32)):
        z, ids = rnd(n, V).to(dtype), torch.randint(0, V, (n, 2), dtype=I32, device="cuda", generator=g)

        def score(z=z, ids=ids, n=n):
            out = {"logprobs": torch.empty(n, 2, device="cuda"), "entropy": torch.empty(n, device="cuda"), "top_ids": torch.empty(n, 9, dtype=I32, device="cuda")}
            return tuple(moev.token_logprobs(z, ids, out).values())
        res.append(score)
    ctx, new = torch.randint(0, 90, (300,), device="cuda", generator=g).to(I32), torch.randint(0, 90, (300,), device="cuda", generator=g).to(I32)
    free, total = torch.randperm(4000, device="cuda", generator=g).to(I32), int(new.sum())
    held = torch.arange(300 * 12, device="cuda").to(I32).view(300, 12)

    def tables():
        table, out = held.clone(), {"cu": t32([0] * 301), "slots": torch.empty(total, dtype=I32, device="cuda"), "positions": torch.empty(total, dtype=I32, device="cuda")}
        moev.build_pages(ctx, new, table, free, 16, out)
        return (table, *out.values())
    return res + [tables]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_calls_at_once_on_streams_of_several_threads():
    calls = programs()
    want = [f() for f in calls]
    torch.cuda.synchronize()
    errors = []

    def work(seed):
        try:
            stream, order = torch.cuda.Stream(), torch.randperm(len(calls), generator=torch.Generator().manual_seed(seed)).tolist()
            with torch.cuda.stream(stream):
                for _ in range(6):
                    got = [(i, calls[i]()) for i in order]
            stream.synchronize()
            errors.extend(i for i, o in got if not same(o, want[i]))
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(s,)) for s in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors


def test_graphs_of_the_same_inputs_replayed_side_by_side():
    calls = programs()[:-1]  # (the tables' tensors are made from host lists: not a thing to capture)
    want = [f() for f in calls]
    torch.cuda.synchronize()
    graphs = []
    for s in range(2):
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            rec = [f() for f in (calls if s == 0 else calls[::-1])]
        graphs.append((stream, graph, rec if s == 0 else rec[::-1]))
    for _ in range(5):
        for stream, graph, _ in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, rec in graphs:
        assert all(same(a, b) for a, b in zip(rec, want))
