"""One token row with strides that would not fit several, through the C entry points."""
import ctypes as C

import pytest
import torch

import block_ref as R
import paper_2607_12696_b200 as moev
from paper_2607_12696_b200.binding import _DraftBatch
from test_gpu_attend_batches import device_batch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_one_row_whatever_its_strides():
    s = R.Setup([37], [1], 16, 2, 4, 64, seed=3, spare=0).poison()
    L = moev.lib()
    got = []
    for stride in (None, 3, -7, 0):
        cache, batch = device_batch(s)
        d = _DraftBatch.from_buffer_copy(batch._c)
        d.n_tokens = 1
        k, v, q, rope = s.nk.cuda(), s.nv.cuda(), s.q.cuda(), s.rope.cuda()
        q_out, out = torch.zeros_like(q), torch.zeros_like(q)
        ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        kv, row = (128, 512) if stride is None else (stride, stride)
        stream = C.c_void_p(torch.cuda.current_stream().cuda_stream)
        assert L.moev_cache_append(C.byref(cache._c), C.byref(d), k.data_ptr(), kv, v.data_ptr(), kv, rope.data_ptr(), rope.shape[0], q.data_ptr(), row, 8,
                                   q_out.data_ptr(), row, stream) == 0
        assert L.moev_cache_attend(C.byref(cache._c), C.byref(d), q_out.data_ptr(), row, 8, 0.125, 0, None, out.data_ptr(), row, None, ws.data_ptr(),
                                   ws.numel(), stream) == 0
        torch.cuda.synchronize()
        got.append((q_out, out, cache.k.view(torch.uint8), cache.v.view(torch.uint8)))
    assert got[0][1].abs().max() > 0
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
