"""The largest numbers of rows: sizes next to the end of 32 bits."""
import pytest
import torch

import paper_2607_12696_b200 as moev

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.fixture(autouse=True)
def memory():
    """These take some 50 GB: nothing of it stays with the allocator."""
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [MOST - 255, MOST])
def test_linear_of_the_most_rows(n):
    codes = torch.zeros(n, 16, dtype=torch.int8, device="cuda")
    ends = [0, 1, 255, 256, 2 ** 30, n - 257, n - 256, n - 2, n - 1]
    for i, at in enumerate(ends):
        codes[at, i] = i + 1
    w = torch.full((1, 16), 3, dtype=torch.int8, device="cuda")
    y = torch.full((n, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    moev.W8Linear(w, torch.ones(1, device="cuda"))((codes, torch.ones(n, device="cuda")), y)
    assert [float(y[at]) for at in ends] == [3.0 * (i + 1) for i in range(len(ends))]
    for at in ends:
        y[at] = 0
    assert int(torch.count_nonzero(y)) == 0


def test_pages_of_the_most_rows():
    """Rows of no sequence up to the last one; as many CTAs as a call of a few rows less takes, so at the same pace (one CTA alone: a hundred times slower)."""
    t = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    ms = {}
    for n in (MOST - 4096, MOST):
        out = {"cu": t([0, 0]), "positions": torch.full((n,), 7, dtype=torch.int32, device="cuda")}
        ms[n] = []
        for _ in range(3):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            moev.build_pages(t([5]), t([9]), t([[3]]), t([1]), 16, out)
            b.record()
            b.synchronize()
            ms[n].append(a.elapsed_time(b))
        pos = out.pop("positions")
        assert pos[:10].tolist() == list(range(5, 14)) + [-1] and int(torch.count_nonzero(pos[9:] + 1)) == 0
        del pos
    assert min(ms[MOST]) < 4 * min(ms[MOST - 4096]), ms
