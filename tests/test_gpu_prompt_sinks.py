"""Sink logits of prompt attention in rows that see nothing, and sinks that are not finite."""
import pytest
import torch

import prompt_ref as R
from test_gpu_prompt_tiles import make, run, within

pytestmark = pytest.mark.gpu

# (n_q, n_k, empty sequences behind, bound on the tokens): keys shared by a cluster, one tile of rows, two tiles
FORMS = {"shared": ([20, 30], [12, 900], 0, 30), "few": ([20, 30], [12, 40], 300, 30), "two": ([20, 30], [12, 900], 160, 1000)}


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_rows_without_keys_have_the_sink_as_it_is_given(form, D):
    n_q, n_k, empty, most = FORMS[form]
    q, k, v, cu, cu_k = make(n_q, n_k, 2, 2, D, empty=empty)
    if form == "few":  # 700 keys of the call or fewer
        k, v = k[:cu_k[-1]], v[:cu_k[-1]]
    sinks = torch.tensor([0.1, -3.7, torch.nan, -torch.inf])
    out, lse = run(q, k, v, cu, cu_k, most, sinks=sinks.cuda())
    assert (out[:8] == 0).all()
    assert torch.equal(lse[:8].cpu().nan_to_num(nan=5.0, neginf=-9.0), sinks.nan_to_num(nan=5.0, neginf=-9.0).expand(8, 4))
    want, want_l, tol, tol_l = R.prompt(q, k, v, cu, cu_k, D ** -0.5, 0, sinks, torch.full(q.shape, 7.0), torch.full(q.shape[:2], 7.0))
    within(lse, want_l, tol_l, "lse")
    within(out, want, tol, "out")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_infinite_sink_leaves_nothing_for_the_keys(form, D):
    n_q, n_k, empty, most = FORMS[form]
    q, k, v, cu, cu_k = make(n_q, n_k, 2, 2, D, empty=empty)
    if form == "few":
        k, v = k[:cu_k[-1]], v[:cu_k[-1]]
    k[cu_k[1] + 5, 1, 2] = torch.nan  # a key of kv head 1 whose scores are NaN: as they are, whatever the sink
    sinks = torch.tensor([torch.inf, 0.3, torch.inf, -torch.inf])
    out, lse = run(q, k, v, cu, cu_k, most, sinks=sinks.cuda())
    want, want_l, tol, tol_l = R.prompt(q, k, v, cu, cu_k, D ** -0.5, 0, sinks, torch.full(q.shape, 7.0), torch.full(q.shape[:2], 7.0))
    assert (want[20:50, 0] == 0).all() and (want_l[20:50, 0] == torch.inf).all() and torch.isnan(want[49, 2]).all()
    within(lse, want_l, tol_l, "lse")
    within(out, want, tol, "out")
