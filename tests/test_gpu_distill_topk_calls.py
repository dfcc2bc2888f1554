"""Calls of the top-log-probability loss as a program makes them: many student rows, one call
behind the other through one workspace, two at once."""
import numpy as np
import pytest
import torch

from helpers import dev, umim
from test_gpu_distill_topk import check, lists, near
from test_gpu_logprobs import logits

pytestmark = pytest.mark.gpu


def i32(a, dv):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).to(dv)


@pytest.mark.parametrize("R", [131072, 131073, 300001, 1500000])
def test_many_student_rows(R):
    """More rows than one pass of the pairs' check marks: every row's gradient, rows in no pair, and a row in two
    pairs wherever it lies."""
    m, dv = umim(), dev()
    V, K, T = 5, 2, 1.0
    N = R * 4 // 5
    g = torch.Generator(device=dv).manual_seed(R)
    x = torch.randn((R, 8), generator=g, device=dv)
    ids, lp = lists(R, 40, K, V, holes=False, mass=0.7)
    sr = torch.randperm(R, generator=g, device=dv)[:N].int()
    tr = torch.randint(0, 40, (N,), generator=g, device=dv).int()
    st = m.new_status(dv)
    top_ids, top_lp = i32(ids, dv), torch.from_numpy(lp).to(dv)
    ws = m.workspace(m.umim_distill_topk_ce_workspace_size(R, N), dv)
    loss, pairs, grad = m.umim_distill_topk_ce(top_ids, top_lp, x, tr, sr, vocab=V, temperature=T, grad_scale=float(N),
                                               workspace_buf=ws, dev_status=st)
    torch.cuda.synchronize()
    m.check_status(st)
    s, at = sr.long(), top_ids[tr.long()].long()
    logq = torch.log_softmax(x[s, :V].double(), 1)
    p = top_lp[tr.long()].double().exp()
    rest = 1 - p.sum(1)
    q_rest = logq.exp().scatter(1, at, 0.0).sum(1)
    want = -(p * logq.gather(1, at)).sum(1) - rest * q_rest.log()
    d = logq.exp() * (1 - rest / q_rest)[:, None]
    d.scatter_(1, at, logq.exp().gather(1, at) - p)
    wgrad = torch.zeros((R, V), dtype=torch.float64, device=dv)
    wgrad[s] = d
    # tens of roundings of values below 1, of |ln q| <= 15, of 1 / q_rest <= e^12
    assert float((pairs.double() - want).abs().max()) <= 64 * 15 * 2.0 ** -24
    assert float(((grad[:, :V].double() - wgrad).abs() / (1 + wgrad.abs())).max()) <= 200 * 2.0 ** -24
    assert abs(float(loss) - float(want.mean())) <= 64 * 15 * 2.0 ** -24
    for a, b in ((0, N - 1), (N // 2, N // 2 + 1)):
        twice = sr.clone()
        twice[b] = twice[a]
        st = m.new_status(dv)
        grad.fill_(3.0)
        m.umim_distill_topk_ce(top_ids, top_lp, x, tr, twice, vocab=V, grad=grad, workspace_buf=ws, dev_status=st)
        torch.cuda.synchronize()
        assert int(st.item()) == 1 and bool((grad == 3).all())
