"""moev_w4_pack: codes are read by 4 bytes, scales one by one; more alignment is not asked for.  No GPU: refused calls only."""
import ctypes as C

import pytest

import paper_2607_12696_b200 as moev
from paper_2607_12696_b200.binding import _Linear
from test_block_args import BASE

L = moev.lib()


@pytest.mark.parametrize("wfmt,codes,scales", [(4, 1, 0), (4, 2, 0), (4, 0, 1), (3, 2, 0)])
def test_pack_refuses_what_it_cannot_read(wfmt, codes, scales):
    assert L.moev_w4_pack(C.byref(_Linear(16, 64, wfmt, 32)), BASE + codes, BASE + scales, BASE, None) == 1
    assert L.moev_w4_pack(C.byref(_Linear(16, 64, wfmt, 32)), BASE, BASE, BASE + 8, None) == 1
