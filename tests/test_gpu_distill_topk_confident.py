"""Distillation from top log probabilities where the student is nearly certain: of
a listed token, of one outside the list, or of the rest as a whole.  Pair losses
and fp32 gradients are exact to the size of what is left, not of 1.

Tolerances (u = 2^-24), with y = (x - max) / T, e = exp(y), L and R the sums of e over the list and the rest, o
that over everything but the largest element.  A sum of exponentials is off by
  E = tol_l + 8 u 64
of itself (test_gpu_logprobs.py; |y| <= 64 where it counts).  p is off by 16 u of itself, p_rest by
16 u (1 - p_max), p_max's complement by both.
  loss      sum p (ln Z - y) + p_rest ln(1 + L / R): terms of one sign, ln Z = ln(1 + o) off by
            E of itself, ln(1 + z) by z's own 2 E of itself
  at the largest element, listed:  (P - p) - P o / Z
  at the other listed ones:        P q - p
  outside:  (e_v / R) (P R / Z - p_rest), or (e_v / R) (sum p - P L / Z) where R > L
"""
import numpy as np
import pytest
import torch

from helpers import dev, umim
from test_gpu_distill_topk_rest import GAPS, padded, sure_rows
from test_gpu_logprobs import TYPES, U, f64, tol_l, within

pytestmark = pytest.mark.gpu


def expected(ids, lam, x, T, tail):
    """One pair, in float64: (loss, its tolerance, gradient times T, its tolerance)."""
    V = len(x)
    E = tol_l(V) + 8 * U * 64
    held = ids >= 0
    ids, lam = ids[held], lam[held].astype(np.float64)
    b = int(lam.argmax())
    if tail:
        left = -np.expm1(lam[b])
        p = np.exp(lam)
        others = np.delete(p, b).sum()
        rest = max(0.0, left - others)
        listed = p.sum()
        P = 1.0 if rest > 0 else listed
    else:
        w = np.exp(lam - lam[b])
        p = w / w.sum()
        others, rest, listed, P = np.delete(p, b).sum(), 0.0, 1.0, 1.0
        left = others
    y = (x - x.max()) / T
    e = np.exp(y)
    j = int(y.argmax())
    outside = np.ones(V, bool)
    outside[ids] = False
    o = np.delete(e, j).sum()
    Z, lz = 1 + o, np.log1p(o)
    L, R = e[ids].sum(), e[outside].sum()
    ln_rest = np.log1p(L / R) if rest > 0 else 0.0
    loss = (p * (lz - y[ids])).sum() + rest * ln_rest
    tol = (p * (E * lz + 4 * U * np.abs(y[ids]) + 16 * U * (lz + np.abs(y[ids])))).sum() \
        + rest * 2 * E * ln_rest + 16 * U * left * ln_rest + 8 * U * loss
    ev = tol_l(V) + 8 * U * (np.abs(y) + 24)       # a single e_v, and over a sum
    pull, dpull = (listed - P * L / Z, listed * 16 * U + P * L / Z * 2 * E) if R > L else \
        (P * R / Z - rest, P * R / Z * 2 * E + 16 * U * left)
    grad = e / R * pull
    gtol = e / R * (np.abs(pull) * ev + dpull)
    grad[ids] = P * e[ids] / Z - p
    gtol[ids] = P * e[ids] / Z * ev[ids] + p * 16 * U
    if j in ids and o < 0.9:
        k = int(np.nonzero(ids == j)[0][0])
        grad[j] = ((others + rest) if k == b else P - p[k]) - P * o / Z
        near = 32 * U * left if p[k] > 0.55 * P else 32 * U
        gtol[j] = near + P * o / Z * 2 * E
    return loss, tol, grad, gtol


def check(ids, lp, x, V, T, tail, dtype):
    """Row k of the student against row k of the teacher's lists."""
    m, dv = umim(), dev()
    R = len(ids)
    rows = torch.arange(R, dtype=torch.int32, device=dv)
    st = m.new_status(dv)
    _, pairs, grad = m.umim_distill_topk_ce(torch.from_numpy(ids).to(dv), torch.from_numpy(lp).to(dv), x.to(dv), rows, rows,
                                            vocab=V, temperature=T, tail=tail, dev_status=st)
    torch.cuda.synchronize()
    m.check_status(st)
    xd, pairs, grad = f64(x)[:, :V], f64(pairs), f64(grad)[:, :V]
    eps = torch.finfo(TYPES[dtype]).eps / 2
    for k in range(R):
        loss, tol, want, gtol = expected(ids[k], lp[k], xd[k], T, tail)
        within(pairs[k:k + 1], [loss], tol, f"pair loss {k}")
        # exponentials below 2^-126 come out as 0; fp32 results below 2^-126 may
        gtol = (gtol + (eps + 4 * U) * np.abs(want) + 2.0 ** -125) / (R * T)
        within(grad[k], want / (R * T), gtol, f"gradient of row {k}")


def lists(seed, x, K, at, gaps):
    """Teacher lists over rows x (float64): `at` first, as sure as `gaps` says, then K - 1 of the row's others, with
    three quarters of what is left."""
    r = np.random.default_rng(seed)
    R, V = x.shape
    ids, lp = np.empty((R, K), np.int32), np.empty((R, K))
    for k in range(R):
        left = 1.0 / (1.0 + np.exp(np.resize(gaps, R)[k]))
        ids[k, 0], lp[k, 0] = at[k], np.log1p(-left)
        if K > 1:
            ids[k, 1:] = r.choice(np.setdiff1d(np.arange(V), at[k]), K - 1, replace=False)
            w = r.random(K - 1) + 0.05
            lp[k, 1:] = np.log(0.75 * left * w / w.sum())
    return ids, lp.astype(np.float32)


SIZES = [(900, 1, "fp32", 1.0), (900, 6, "fp32", 0.7), (20011, 40, "fp32", 1.0), (20011, 128, "bf16", 1.0), (70001, 64, "fp32", 1.3)]


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("V,K,dtype,T", SIZES)
def test_sure_of_the_teachers_best(V, K, dtype, T, tail):
    R = 14
    x, at = sure_rows(V + K, R, V, GAPS)
    ids, lp = lists(V, x, K, at, GAPS[::-1])
    check(ids, lp, padded(T * x, dtype), V, T, tail, dtype)


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("V,K,dtype,T", SIZES[1:])
def test_sure_of_another_listed_token(V, K, dtype, T, tail):
    R = 14
    x, at = sure_rows(V + K, R, V, GAPS)
    other = (at + 7) % V
    ids, lp = lists(V, x, K, other, GAPS)
    for k in range(R):
        if at[k] not in ids[k]:
            ids[k, -1] = at[k]
    check(ids, lp, padded(T * x, dtype), V, T, tail, dtype)


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("V,K,dtype,T", SIZES)
def test_sure_of_a_token_outside_the_list(V, K, dtype, T, tail):
    R = 14
    x, at = sure_rows(V + K, R, V, GAPS)
    ids, lp = lists(V, x, K, (at + 7) % V, GAPS)
    for k in range(R):   # not in the list
        ids[k] = np.where(ids[k] == at[k], (at[k] + 8) % V, ids[k])
        if len(set(ids[k])) < K:
            ids[k, 1:] = np.setdiff1d(np.arange(V), [at[k], ids[k, 0]])[:K - 1]
    check(ids, lp, padded(T * x, dtype), V, T, tail, dtype)


@pytest.mark.parametrize("V,K,dtype,T", SIZES)
def test_both_sure_of_the_rest(V, K, dtype, T):
    """A list of unlikely tokens: the teacher's and the student's mass lies outside it, on no token in particular."""
    R = 14
    r = np.random.default_rng(V)
    x = 1.5 * r.standard_normal((R, V))
    ids = np.stack([r.choice(V, K, replace=False) for _ in range(R)]).astype(np.int32)
    # the list's share: about e^-gap, of both
    lse = np.log(np.exp(x).sum(1))
    gap = np.resize(GAPS, R)
    w = r.random((R, K)) + 0.05
    lp = np.log(w / w.sum(1, keepdims=True)) - gap[:, None]
    np.put_along_axis(x, ids.astype(np.int64), lp + lse[:, None] + 0.3 * r.standard_normal((R, K)), 1)
    check(ids, lp.astype(np.float32), padded(T * x, dtype), V, T, True, dtype)


@pytest.mark.parametrize("tail", [True, False])
def test_equal_largest_elements(tail):
    """Two or three of the largest: listed both, one outside, in one warp's stretch and in others'."""
    V, K, R = 20011, 12, 6
    x, at = sure_rows(5, R, V, [12.0])
    ids, lp = lists(6, x, K, at, [3.0])
    for k in range(R):
        second = int(ids[k, 1]) if k % 3 == 0 else (at[k] + (1 if k % 3 == 1 else V // 2)) % V
        x[k, second] = x[k, at[k]]
        if k == 3:
            x[k, ids[k, 2]] = x[k, at[k]]
    check(ids, lp, padded(x, "fp32"), V, 1.0, tail, "fp32")
