"""What a caller learns of a time-out of the attention kernel (outputs undefined): nothing else may hide it."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def result():
    from paper_2607_12696_b200.build import build
    build()
    p = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "attend_status_child.py")], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stdout[-2000:] + p.stderr[-4000:]
    return json.loads([l for l in p.stdout.splitlines() if l.startswith("RESULT ")][-1][len("RESULT "):])


def test_a_time_out_stays_in_the_status_word_beside_a_rejected_sequence(result):
    assert result["rejected"] == [[0, 1], [0, 4], [0, 1]]


def test_blocks_report_a_time_out_of_their_attention(result):
    """moev_status_sync says so, with and without a status word of the batch."""
    quiet, quiet_word, late, late_word = result["blocks"]
    assert quiet == [0, 0, None] and quiet_word == [0, 0, 0]
    assert late[0] != 0 and late == [late[0], 0, None] and late_word == [late[0], 0, 4]
