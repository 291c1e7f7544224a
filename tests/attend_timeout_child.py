"""Child process of test_gpu_attend_timeout.py: the test-hook build of the library, whose attention kernel can be made to
wait for a tile that never comes.  Prints one JSON object."""
import ctypes as C
import json
import os
import sys
import time

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path[:0] = [ROOT, os.path.join(ROOT, "tests")]

import torch  # noqa: E402

import block_ref as R  # noqa: E402
import paper_2607_12696_b200.binding as binding  # noqa: E402
from paper_2607_12696_b200.build import TEST_LIB  # noqa: E402

binding._LIB_PATH = TEST_LIB  # before the first lib() call; the calls below go through ctypes, not the compiled checks


def main():
    L = binding.lib()
    L.moev_test_withhold_attend.restype = C.c_int32
    res = {}
    for D, rep, n in ((64, 2, 3), (128, 8, 4), (128, 16, 4), (64, 16, 20)):  # one case per tile of rows
        s = R.Setup([700, 40], [n, 1], 64, 2, rep, D, True, seed=D + rep).poison()
        dev = {k: getattr(s, k).cuda().contiguous() for k in ("k", "v", "ks", "vs", "q", "table", "parent")}
        cu, ctx = torch.tensor(s.cu, dtype=torch.int32).cuda(), torch.tensor(s.ctx, dtype=torch.int32).cuda()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        c = binding._KvCache(s.n_pages, 64, 2, D, *[dev[k].data_ptr() for k in ("k", "v", "ks", "vs")])
        d = binding._DraftBatch(2, s.T, s.max_drafts, s.max_len, s.cols, cu.data_ptr(), ctx.data_ptr(), dev["table"].data_ptr(),
                                dev["parent"].data_ptr(), status.data_ptr())
        heads = 2 * rep
        size = L.moev_cache_attend_workspace(C.byref(c), C.byref(d), heads, 0)
        ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")

        def call():
            out = torch.zeros(s.T, heads, D, dtype=torch.bfloat16, device="cuda")
            t0 = time.perf_counter()
            st = L.moev_cache_attend(C.byref(c), C.byref(d), dev["q"].data_ptr(), heads * D, heads, D ** -0.5, 0, None, out.data_ptr(), heads * D, None,
                                     ws.data_ptr(), size, C.c_void_p(torch.cuda.current_stream().cuda_stream))
            torch.cuda.synchronize()
            got = int(status)
            status.zero_()
            return out, st, got, time.perf_counter() - t0

        ref = s.attend()[0][:s.cu[-1]].cuda()
        err = lambda o: float((o[:s.cu[-1]].double() - ref).abs().max() / ref.abs().max())  # noqa: E731
        before = call()
        L.moev_test_withhold_attend(1)
        held = call()
        L.moev_test_withhold_attend(0)
        after = call()
        res[f"D{D}_rows{n * rep}"] = {"launch": [x[1] for x in (before, held, after)], "status": [x[2] for x in (before, held, after)], "wall_s": held[3],
                                      "err": [err(before[0]), err(after[0])]}
    print("RESULT " + json.dumps(res))


if __name__ == "__main__":
    main()
