"""Child process of test_gpu_attend_status.py, on the test-hook build: a time-out of the attention kernel beside a rejected
sequence, and inside moev_verify_blocks.  Prints one JSON object."""
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path[:0] = [ROOT, os.path.join(ROOT, "tests")]

import ctypes as C  # noqa: E402

import torch  # noqa: E402

import block_ref as R  # noqa: E402
import paper_2607_12696_b200 as moev  # noqa: E402
import paper_2607_12696_b200.binding as binding  # noqa: E402
from paper_2607_12696_b200.build import TEST_LIB  # noqa: E402

binding._LIB_PATH = TEST_LIB  # before the first lib() call; nothing here goes through the compiled checks


def rejected_and_timed_out(L, withhold):
    """Three sequences, the second one behind the call's bounds; many tiles, so that a second kernel joins the parts."""
    s = R.Setup([700, 30, 900], [3, 2, 3], 64, 2, 4, 64, True, seed=1).poison()
    cache = moev.KvCache(s.k.cuda().contiguous(), s.v.cuda().contiguous(), s.ks.cuda(), s.vs.cuda())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    batch = moev.DraftBatch(i32(s.cu), i32([700, 5000, 900]), s.table.cuda(), s.max_drafts, s.max_len, s.parent.cuda(), status)
    d = binding._DraftBatch.from_buffer_copy(batch._c)
    d.n_tokens = s.T
    heads = 8
    ws = moev.cache_attend_workspace(cache, batch, heads)
    q, out = s.q.cuda(), torch.zeros(s.T, heads, 64, dtype=torch.bfloat16, device="cuda")
    L.moev_test_withhold_attend(withhold)
    st = L.moev_cache_attend(C.byref(cache._c), C.byref(d), q.data_ptr(), heads * 64, heads, 0.125, 0, None, out.data_ptr(), heads * 64, None,
                             ws.data_ptr(), ws.numel(), C.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    L.moev_test_withhold_attend(0)
    return [st, int(status)]


def blocks(L, withhold, with_status):
    import test_gpu_blocks as B
    s = B.setup()
    m = B.Model(2, s, H=704, I=320, E=32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda") if with_status else None
    m.batch = moev.DraftBatch(m.batch.cu, m.batch.ctx_len, m.batch.page_table, m.batch.max_drafts, m.batch.max_len, m.batch.parent, status)
    L.moev_test_withhold_attend(withhold)
    m.v.verify_blocks(m.blocks, m.batch, m.h.clone(), m.n_heads, m.outs(), rope=m.rope)
    torch.cuda.synchronize()
    L.moev_test_withhold_attend(0)
    codes = []
    for _ in range(2):  # the second read finds the word cleared
        try:
            m.v.status_sync()
            codes.append(0)
        except moev.MoevError as e:
            codes.append(e.status)
    m.v.close()
    return codes + [int(status) if with_status else None]


def main():
    L = binding.lib()
    L.moev_test_withhold_attend.restype = C.c_int32
    res = {"rejected": [rejected_and_timed_out(L, w) for w in (0, 1, 0)],
           "blocks": [blocks(L, w, st) for w in (0, 1) for st in (False, True)]}
    print("RESULT " + json.dumps(res))


if __name__ == "__main__":
    main()
