"""Pages that a window has left behind: their entries in the page table are not looked at."""
import pytest
import torch

import block_ref as R
import paper_2607_12696_b200 as moev
from test_gpu_attend_batches import check, device_batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("gone", [-1, 10 ** 6])
def test_pages_in_front_of_the_window_may_be_gone(page, tree, gone):
    """A page of which no draft sees a key may have been given back: its entry is not looked at, wherever tiles begin."""
    for ctx, window in ((150, 20), (300, 45), (128, 1), (127, 2), (400, 130), (77, 16)):
        s = R.Setup([ctx], [3], page, 1, 2, 64, tree, seed=ctx).poison()
        cache, batch = device_batch(s)
        want = moev.cache_attend(cache, batch, s.q.cuda(), window=window).clone()
        batch.page_table[0, :(ctx + 1 - window) // page] = gone
        got = moev.cache_attend(cache, batch, s.q.cuda(), window=window)
        assert int(batch.status) == 0 and torch.equal(got, want)
        check(s, window=window)
        if (ctx + 1 - window) % page:  # the first page that is seen is looked at
            batch.page_table[0, (ctx + 1 - window) // page] = gone
            moev.cache_attend(cache, batch, s.q.cuda(), window=window)
            assert int(batch.status) == 2
