"""Windows of prompt attention as wide as the keys and wider, up to the largest integer."""
import pytest
import torch

from test_gpu_prompt_tiles import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q,n_k,rep,empty,most", [([20], [10], 2, 300, 20), ([20, 9], [10, 30], 2, 0, 30), ([300, 20], [100, 900], 1, 160, 1000)])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 64, 1811, 1810, 1000, 910, 840, 810])
def test_window_wider_than_the_keys(window, n_q, n_k, rep, empty, most, D):
    """Rows of negative positions beside ones that see keys: the largest windows hide nothing (keys of the call: 810, 840, 1800)."""
    check(*make(n_q, n_k, 1, rep, D, seed=2, empty=empty), most, window=window)
