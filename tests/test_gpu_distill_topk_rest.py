"""Distillation from top log probabilities where the teacher is nearly certain of
one token: p_rest keeps its digits, whatever is left of 1.

Tolerances (u = 2^-24).  p_rest is (1 - p_max) - others: expm1f is off by 2 u of
1 - p_max, each other p by 4 u of itself (its exponential), their sum by 9 u (four terms a
lane, five steps over the lanes), the difference by u; and others <= 1 - p_max.
So p_rest is off by 16 u (1 - p_max).  An element outside the list has the gradient
q_v (P - p_rest / q_rest) / (N T), with q_v = e_v / Z and q_v / q_rest = e_v / R: both of these are off by
e_v's 8 u (|ln q_v| + 24) and by their sum's tol_l, as in test_gpu_distill_topk.py.
"""
import numpy as np
import pytest
import torch

from helpers import dev, umim
from oracle import logprobs as OL
from test_gpu_logprobs import TYPES, U, f64, tol_l, within

pytestmark = pytest.mark.gpu


def sure_rows(seed, R, V, gaps, std=1.5):
    """[R][V] float64 logits, in each row one element `gap` nats above the sum of the others; and its id."""
    r = np.random.default_rng(seed)
    x = std * r.standard_normal((R, V))
    at = r.integers(0, V, R)
    x[np.arange(R), at] = -np.inf
    m = x.max(1)
    x[np.arange(R), at] = m + np.log(np.exp(x - m[:, None]).sum(1)) + np.resize(gaps, R)
    return x, at


def best(x, K):
    """The K best ids of float64 rows and their log probabilities, as fp32."""
    ids = np.argsort(-x, axis=1, kind="stable")[:, :K]
    m = x.max(1, keepdims=True)
    e = np.exp(x - m)
    e[np.arange(len(x)), ids[:, 0]] = 0.0
    lp = np.take_along_axis(x - m, ids, 1) - np.log1p(e.sum(1))[:, None]
    return ids.astype(np.int32), lp.astype(np.float32)


def padded(x, dtype):
    out = torch.full((x.shape[0], -(-x.shape[1] // 8) * 8), float("nan"))
    out[:, :x.shape[1]] = torch.from_numpy(x.astype(np.float32))
    return out.to(TYPES[dtype])


def one_minus_max(lam):
    """1 - p_max and the other entries' sum, of fp32 log probabilities in descending order."""
    lam = lam.astype(np.float64)
    return -np.expm1(lam[0]), np.exp(lam[1:]).sum()


GAPS = [4.0, 6.0, 8.0, 10.0, 12.0, 14.0, 16.0]


@pytest.mark.parametrize("source", ["cache", "float64"])
@pytest.mark.parametrize("V,R,K,dtype,T", [(700, 14, 5, "fp32", 1.0), (5000, 21, 20, "fp32", 1.0), (5000, 21, 64, "bf16", 1.0),
                                           (20011, 300, 128, "fp32", 1.3), (128256, 7, 64, "fp32", 1.0)])
def test_a_small_rest_keeps_its_digits(source, V, R, K, dtype, T):
    m, dv = umim(), dev()
    teacher, at = sure_rows(V + K, R, V, GAPS)
    r = np.random.default_rng(K)
    student = T * (teacher + 0.3 * r.standard_normal((R, V)))
    st = m.new_status(dv)
    if source == "cache":
        c = m.umim_token_logprobs(padded(teacher, "fp32").to(dv), n_top=K, vocab=V, dev_status=st)
        top_ids, top_lp = c["top_ids"], c["top_logprobs"]
        ids, lp = top_ids.cpu().numpy(), top_lp.cpu().numpy()
    else:
        ids, lp = best(teacher, K)
        top_ids, top_lp = torch.from_numpy(ids).to(dv), torch.from_numpy(lp).to(dv)
    assert (ids[:, 0] == at).all()
    x = padded(student, dtype)
    rows = torch.arange(R, dtype=torch.int32, device=dv)
    _, _, grad = m.umim_distill_topk_ce(top_ids, top_lp, x.to(dv), rows, rows, vocab=V, temperature=T, dev_status=st)
    torch.cuda.synchronize()
    m.check_status(st)
    got, xd = f64(grad)[:, :V], f64(x)[:, :V]
    eps = torch.finfo(TYPES[dtype]).eps / 2
    for k in range(R):
        left, others = one_minus_max(lp[k])
        rest = left - others
        assert rest > 0
        y = (xd[k] - xd[k].max()) / T
        e = np.exp(y)
        outside = np.ones(V, bool)
        outside[ids[k]] = False
        q, share = e / e.sum(), e / e[outside].sum()        # q_v, and q_v / q_rest
        want = (q - rest * share) / (R * T)
        off = 2 * tol_l(V) + 8 * U * (np.abs(np.log(q)) + 24)
        tol = ((q + rest * share) * off + share * 16 * U * left) / (R * T) + (eps + 4 * U) * np.abs(want)
        # an exponential below 2^-126 comes out as 0
        tol = tol + 2.0 ** -125 / (R * T)
        within(got[k][outside], want[outside], tol[outside], f"outside the list of row {k}")


@pytest.mark.parametrize("mask", ["lowest", "-inf"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_rest_of_rounding_counts_only_where_the_student_has_one(dtype, mask):
    """Teacher and student under one mask, by the type's lowest value or -inf, the list complete: what rounding
    leaves of 1 is no rest, whose cost would be p_rest times the mask's depth.  A student without
    the mask has a rest, and is measured by what the list says."""
    m, dv = umim(), dev()
    V, R, K = 5000, 12, 24
    r = np.random.default_rng(3)
    allowed = r.permutation(V)[:20]
    blocked = torch.from_numpy(np.setdiff1d(np.arange(V), allowed))
    fill = torch.finfo(TYPES[dtype]).min if mask == "lowest" else -float("inf")
    t, x = (padded(2.0 * r.standard_normal((R, V)), dtype) for _ in range(2))
    t[:, blocked] = -float("inf")
    x[:6, blocked] = fill
    st = m.new_status(dv)
    c = m.umim_token_logprobs(t.to(dv), n_top=K, vocab=V, dev_status=st)
    ids, lp = c["top_ids"].cpu().numpy(), c["top_logprobs"].cpu().numpy()
    rows = torch.arange(R, dtype=torch.int32, device=dv)
    loss, pairs, grad = m.umim_distill_topk_ce(c["top_ids"], c["top_logprobs"], x.to(dv), rows, rows, vocab=V,
                                               dev_status=st)
    torch.cuda.synchronize()
    m.check_status(st)
    want, wpairs, wgrad = OL.topk_ce(ids, lp, f64(x)[:, :V], np.arange(R), np.arange(R))
    assert np.isfinite(wpairs).all() and wpairs.max() < 40
    # |ln q| below 40 everywhere that counts, p off by 16 u and ln q by tol_l + 8 u |ln q|
    within(f64(pairs), wpairs, 2 * (tol_l(V) + 8 * U * 40) + 40 * 40 * U, "pair losses")
    eps = torch.finfo(TYPES[dtype]).eps / 2
    within(f64(grad)[:, :V], wgrad, (eps + 4 * U) * np.abs(wgrad) + (4 * tol_l(V) + 800 * U) / R, "gradient")
    assert bool((grad[:6, blocked.to(dv)] == 0).all())


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("K", [1, 20, 33, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_teacher_row_without_a_distribution_is_not_lost(bad, K, tail):
    """NaN or +inf among the teacher's logits: the cache says so, and the pair's loss and gradient are NaN, as are those
    of a list with NaN at an id.  A row left out, and one whose ids are -1 whatever stands beside, ask nothing."""
    m, dv = umim(), dev()
    V, R = 3000, 6
    r = np.random.default_rng(K)
    t, x = padded(2.0 * r.standard_normal((R, V)), "bf16"), padded(2.0 * r.standard_normal((R, V)), "fp32")
    t[1, V - 1] = bad
    tok = torch.tensor([0, 0, -1, 0, 0, 0], dtype=torch.int32, device=dv)
    st = m.new_status(dv)
    c = m.umim_token_logprobs(t.to(dv), tok, n_top=K, vocab=V, dev_status=st)
    ids, lp = c["top_ids"], c["top_logprobs"]
    ids[3], lp[3] = -1, 0.25
    lp[3, 0] = float("nan") if K > 1 else 0.25
    lp[4, K // 2] = float("nan")
    x[5, :V] = -float("inf")
    rows = torch.arange(R, dtype=torch.int32, device=dv)
    tr = torch.tensor([0, 1, 2, 3, 4, 1], dtype=torch.int32, device=dv)   # the last: a student row of -inf only
    loss, pairs, grad = m.umim_distill_topk_ce(ids, lp, x.to(dv), tr, rows, vocab=V, tail=tail, dev_status=st)
    torch.cuda.synchronize()
    m.check_status(st)
    grad = grad[:, :V]
    for k in (1, 4, 5):
        assert bool(pairs[k].isnan()) and bool(grad[k].isnan().all()), k
    for k in (2, 3):
        assert float(pairs[k]) == 0 and bool((grad[k] == 0).all()), k
    assert bool(pairs[0].isfinite()) and bool(grad[0].isfinite().all()) and bool(loss.isnan().all())
    want, wpairs, wgrad = OL.topk_ce(ids.cpu().numpy(), lp.cpu().numpy(), f64(x)[:, :V], tr.cpu().numpy(), np.arange(R), 1.0,
                                     tail)
    assert np.isnan(want) and np.array_equal(np.isnan(wpairs), np.isnan(f64(pairs)))
    assert np.array_equal(np.isnan(wgrad), np.isnan(f64(grad)))
