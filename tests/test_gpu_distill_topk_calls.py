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


def cases(dv, V, K, shapes, dtype="bf16"):
    """Student rows, lists and pairs of calls that differ in all of them, on the host and as arguments."""
    out = []
    for seed, (R, N) in enumerate(shapes):
        r = np.random.default_rng(100 + seed)
        ids, lp = lists(seed, 30, K, V, mass=0.6 + 0.05 * seed)
        tr, sr = r.integers(0, 30, N), r.permutation(R)[:N]
        x = near(logits(seed, R, V, dtype), ids, lp, tr, sr, 1.0)
        out.append(((ids, lp, x, tr, sr), (i32(ids, dv), torch.from_numpy(lp).to(dv), x.to(dv), i32(tr, dv), i32(sr, dv))))
    return out


# rows, pairs: started beside the plan (few rows a cluster) and behind it, in turn; no pairs; one
SHAPES = [(40, 33), (1300, 1201), (3, 2), (900, 0), (200, 1), (1300, 1300), (300, 150), (40, 40)]


@pytest.mark.parametrize("V", [300, 20011])
def test_one_call_behind_the_other_through_one_workspace(V):
    """Each call's plan writes over what the call before it reads: no synchronisation stands between them but their own."""
    m, dv = umim(), dev()
    K = 24
    todo = cases(dv, V, K, SHAPES)
    ws = m.workspace(m.umim_distill_topk_ce_workspace_size(1300, 1300), dv)
    alone = []
    for (ids, lp, x, tr, sr), args in todo:
        st = m.new_status(dv)
        alone.append(m.umim_distill_topk_ce(*args, vocab=V, dev_status=st))
        torch.cuda.synchronize()
        m.check_status(st)
        if len(sr) <= 200:
            check(alone[-1], ids, lp, x, V, tr, sr, 1.0, True, "bf16")
    order = list(range(len(todo))) * 3 + list(range(len(todo)))[::-1] + [1, 2] * 5 + [0, 7] * 5
    outs = [(torch.full((1,), 9.0, device=dv), torch.full_like(alone[k][1], 9.0), torch.full_like(alone[k][2], 9.0))
            for k in order]
    st = m.new_status(dv)
    torch.cuda.synchronize()
    for k, (loss, pairs, grad) in zip(order, outs):
        m.umim_distill_topk_ce(*todo[k][1], vocab=V, workspace_buf=ws, loss=loss, pair_loss=pairs, grad=grad, dev_status=st)
    torch.cuda.synchronize()
    m.check_status(st)
    for k, (loss, pairs, grad) in zip(order, outs):
        N = len(todo[k][0][4])
        assert torch.equal(loss, alone[k][0]) and torch.equal(pairs[:N], alone[k][1][:N]), k
        assert torch.equal(grad[:, :V], alone[k][2][:, :V]), k


def test_the_students_rows_written_just_before_the_call():
    """The kernel that is started early loads its first row before it waits for the plan: not before what precedes the call."""
    m, dv = umim(), dev()
    V, K = 30000, 20
    todo = cases(dv, V, K, [(40, 40), (40, 37), (40, 40)], "fp32")
    alone = [m.umim_distill_topk_ce(*args, vocab=V) for _, args in todo]
    ws = m.workspace(m.umim_distill_topk_ce_workspace_size(40, 40), dv)
    x, sr = torch.zeros_like(todo[0][1][2]), torch.zeros(40, dtype=torch.int32, device=dv)
    outs = []
    torch.cuda.synchronize()
    for _ in range(10):
        for _, (ids, lp, xs, tr, s) in todo:
            x.copy_(xs)
            sr[:len(s)].copy_(s)
            outs.append(m.umim_distill_topk_ce(ids, lp, x, tr, sr[:len(s)], vocab=V, workspace_buf=ws))
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        want = alone[i % 3]
        assert torch.equal(o[0], want[0]) and torch.equal(o[1], want[1]) and torch.equal(o[2][:, :V], want[2][:, :V]), i


def test_two_calls_at_once():
    m, dv = umim(), dev()
    V, K = 20011, 24
    todo = cases(dv, V, K, [(700, 650), (40, 33)])
    alone = [m.umim_distill_topk_ce(*args, vocab=V) for _, args in todo]
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    ws = [m.workspace(m.umim_distill_topk_ce_workspace_size(700, 650), dv) for _ in streams]
    torch.cuda.synchronize()
    outs = []
    for i in range(12):
        for j, s in enumerate(streams):
            k = (i + j) % 2
            outs.append((k, m.umim_distill_topk_ce(*todo[k][1], vocab=V, workspace_buf=ws[j], stream=s)))
    torch.cuda.synchronize()
    for k, o in outs:
        N = len(todo[k][0][4])
        assert torch.equal(o[0], alone[k][0]) and torch.equal(o[1][:N], alone[k][1][:N])
        assert torch.equal(o[2][:, :V], alone[k][2][:, :V])
