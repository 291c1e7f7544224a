"""The bounded waits of the attention kernel, made to run out.

In the test-hook build (two milliseconds per wait) its loader can be told to leave out the last V tile.  The softmax warps'
wait for it ends, they raise the CTA's abort flag, the MMA issuer leaves and waits for what it issued, copies in flight land,
tensor memory is given back and the status word says so.  Nothing faults or spins without a bound; the next call is right."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_attention_waits_run_out_and_the_next_call_is_right():
    from paper_2607_12696_b200.build import build
    build()
    p = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "attend_timeout_child.py")], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stdout[-2000:] + p.stderr[-4000:]
    res = json.loads([l for l in p.stdout.splitlines() if l.startswith("RESULT ")][-1][len("RESULT "):])
    assert len(res) == 4
    for name, r in res.items():
        assert r["launch"] == [0, 0, 0] and r["status"] == [0, 4, 0], name
        assert r["wall_s"] < 5.0 and max(r["err"]) < 2e-2, name
