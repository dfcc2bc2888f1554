"""Pins of the oracle's log probabilities, their gradient and the soft-target
cross-entropy from top log probabilities: torch's log_softmax, sort and autograd
in float64, App. F's loss over the whole vocabulary, and closed forms."""
import numpy as np
import pytest
import torch

from oracle.distill import soft_ce
from oracle.logprobs import token_logprobs, token_logprobs_grad, topk_ce


def rows(seed, R=7, V=61, levels=None):
    r = np.random.default_rng(seed)
    x = 3.0 * r.standard_normal((R, V))
    return r, (np.round(x * levels) / levels if levels else x)


@pytest.mark.parametrize("T", [1.0, 0.6, 3.0])
def test_log_probabilities_are_log_softmax(T):
    r, x = rows(1)
    tok = r.integers(0, 61, 7)
    got = token_logprobs(x, tok, T, 61)
    want = torch.log_softmax(torch.from_numpy(x) / T, 1).numpy()
    assert np.allclose(got["logprobs"], want[np.arange(7), tok], atol=1e-13)
    assert np.allclose(got["entropy"], -(np.exp(want) * want).sum(1), atol=1e-13)
    m, l = got["stats"].T
    assert np.allclose(m / T + l, torch.logsumexp(torch.from_numpy(x) / T, 1).numpy(), atol=1e-13)
    assert np.allclose(np.take_along_axis(want, got["top_ids"], 1), got["top_logprobs"], atol=1e-13)
    assert (np.diff(got["top_logprobs"], axis=1) <= 0).all()


def test_alternatives_break_ties_by_the_lowest_id():
    _, x = rows(2, levels=1)   # whole numbers: many equal logits
    got = token_logprobs(x, n_top=20)["top_ids"]
    want = torch.from_numpy(x).sort(dim=1, descending=True, stable=True)[1][:, :20].numpy()
    assert (got == want).all()


def test_rows_without_a_distribution():
    x = np.array([[-np.inf] * 4, [1.0, np.nan, 0.0, 0.0], [np.inf, 0.0, 0.0, 0.0], [0.0, -np.inf, 0.0, -np.inf],
                  [5.0, 6.0, 7.0, 8.0]])
    tok = np.array([1, 0, 0, 1, -1])
    got = token_logprobs(x, tok, 1.0, 3)
    assert got["logprobs"][0] == -np.inf and got["entropy"][0] == 0 and got["stats"][0].tolist() == [-np.inf, 0.0]
    assert np.isnan(got["logprobs"][1:3]).all() and np.isnan(got["stats"][1:3]).all()
    assert (got["top_ids"][:3] == -1).all() and np.isnan(got["top_logprobs"][1:3]).all()
    assert got["logprobs"][3] == -np.inf and got["top_ids"][3].tolist() == [0, 2, -1]
    assert np.isclose(got["entropy"][3], np.log(2.0))
    assert got["logprobs"][4] == 0 and (got["stats"][4] == 0).all() and (got["top_ids"][4] == -1).all()
    grad = token_logprobs_grad(x, tok, np.ones(5), np.ones(5))
    assert (grad[[0, 4]] == 0).all() and np.isnan(grad[1:3]).all() and grad[3, 1] == 1.0


@pytest.mark.parametrize("g_on,h_on,T", [(True, False, 1.0), (False, True, 0.7), (True, True, 2.0)])
def test_gradient_is_autograd(g_on, h_on, T):
    r, x = rows(3)
    tok, g, h = r.integers(0, 61, 7), r.standard_normal(7), r.standard_normal(7)
    t = torch.from_numpy(x).requires_grad_()
    logp = torch.log_softmax(t / T, 1)
    f = 0.0
    if g_on:
        f = f + (torch.from_numpy(g) * logp[torch.arange(7), torch.from_numpy(tok)]).sum()
    if h_on:
        f = f - (torch.from_numpy(h)[:, None] * logp.exp() * logp).sum()
    f.backward()
    got = token_logprobs_grad(x, tok, g if g_on else None, h if h_on else None, T)
    assert np.allclose(got, t.grad.numpy(), atol=1e-13)


def test_gradient_is_the_difference_quotient():
    r, x = rows(4, R=2, V=9)
    tok, g, h, d = np.array([3, 8]), r.standard_normal(2), r.standard_normal(2), 1e-6
    f = lambda y: (lambda o: (g * o["logprobs"] + h * o["entropy"]).sum())(token_logprobs(y, tok, 1.3))
    got = token_logprobs_grad(x, tok, g, h, 1.3)
    for i in np.ndindex(x.shape):
        e = np.zeros(x.shape)
        e[i] = d
        assert abs((f(x + e) - f(x - e)) / (2 * d) - got[i]) < 1e-8


def lists(r, R_T, K, V, mass=0.9):
    ids = np.stack([r.permutation(V)[:K] for _ in range(R_T)])
    w = r.random((R_T, K)) + 0.01
    return ids, np.log(mass * w / w.sum(1, keepdims=True))


@pytest.mark.parametrize("tail", [True, False])
def test_full_lists_give_the_full_vocabulary_loss(tail):
    """Every id listed with the teacher's log-softmax: the soft cross-entropy over the whole vocabulary."""
    r, x = rows(5, V=40)
    teacher = 2.0 * r.standard_normal((5, 40))
    got = token_logprobs(teacher, n_top=40)
    tr, sr = [4, 0, 2], [1, 6, 3]
    loss, _, grad = topk_ce(got["top_ids"], got["top_logprobs"], x, tr, sr, 1.0, tail)
    want, wgrad = soft_ce(teacher, x, tr, sr, eps=0.0)
    assert np.isclose(loss, want, atol=1e-12) and np.allclose(grad, wgrad, atol=1e-12)


@pytest.mark.parametrize("tail,T", [(True, 1.0), (True, 1.7), (False, 0.8)])
def test_topk_gradient_is_autograd(tail, T):
    r, x = rows(6)
    ids, lp = lists(r, 6, 8, 61)
    ids[2, 5:] = -1
    tr, sr = np.array([2, 5, 0]), np.array([0, 3, 6])
    t = torch.from_numpy(x).requires_grad_()
    total = 0.0
    for a, b in zip(tr, sr):
        keep = ids[a] >= 0
        p = torch.from_numpy(np.exp(lp[a][keep]))
        q = torch.softmax(t[b] / T, 0)
        if not tail:
            p = p / p.sum()
        total = total - (p * q[torch.from_numpy(ids[a][keep])].log()).sum()
        if tail:
            out = torch.ones(61, dtype=torch.bool)
            out[torch.from_numpy(ids[a][keep])] = False
            total = total - (1 - p.sum()) * q[out].sum().log()
    (total / 3).backward()
    loss, pairs, grad = topk_ce(ids, lp, x, tr, sr, T, tail)
    assert np.isclose(loss, total.item() / 3) and np.isclose(pairs.mean(), loss)
    assert np.allclose(grad, t.grad.numpy(), atol=1e-13)


def test_teacher_rows_without_entries_and_equal_distributions():
    r, x = rows(7, R=3, V=12)
    empty = np.full((1, 4), -1), np.zeros((1, 4))
    for tail in (True, False):
        loss, pairs, grad = topk_ce(*empty, x, [0], [1], 1.0, tail)
        assert abs(loss) < 1e-12 and np.allclose(grad, 0, atol=1e-15)
    # the student's own top entries: the gradient vanishes with the tail
    own = token_logprobs(x, n_top=5)
    _, _, grad = topk_ce(own["top_ids"], own["top_logprobs"], x, [0, 1, 2], [0, 1, 2], 1.0, True)
    assert np.allclose(grad, 0, atol=1e-15)
    assert topk_ce(*empty, x, [], [], 1.0, True)[0] == 0.0
