"""Several host threads whose first calls come at the same time, each on its own stream: what one thread alone gets."""
import threading

import pytest
import torch

import block_ref as R
import paper_2607_12696_b200 as moev
from test_gpu_attend_batches import device_batch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_threads_with_a_stream_each():
    s = R.Setup([300, 20], [3, 2], 32, 2, 4, 64, True, seed=4).poison()
    g = torch.Generator().manual_seed(1)
    codes, scales = torch.randint(0, 256, (96, 128), generator=g, dtype=torch.uint8).cuda(), torch.full((96, 8), 0.01, dtype=BF16, device="cuda")
    x, w = torch.randn(5, 256, generator=g).to(BF16).cuda(), torch.ones(256, dtype=BF16, device="cuda")
    q = s.q.cuda()
    lin = moev.W4Linear(codes, scales)
    cache, batch = device_batch(s)
    torch.cuda.synchronize()
    start, got, failed = threading.Barrier(6), [None] * 6, []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait()
                for _ in range(20):
                    y = moev.add_rmsnorm(x, w, {"y": torch.empty_like(x)})["y"]
                    got[i] = (lin(y), moev.cache_attend(cache, batch, q))
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(6)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not failed
    want = (lin(moev.add_rmsnorm(x, w, {"y": torch.empty_like(x)})["y"]), moev.cache_attend(cache, batch, q))
    assert all(torch.equal(a, b) for one in got for a, b in zip(one, want))
