"""Log probabilities of given tokens, entropy, alternatives, their gradient, and
the soft-target cross-entropy from a teacher's top log probabilities, of the
oracle (test infrastructure only), in float64.

With p = softmax(x / T) over a row x:
  logprob = ln p_t,  H = -sum p ln p (0 ln 0 = 0),
  stats   = (max x, ln sum exp((x - max x) / T));
  alternatives: the logits above -inf in descending order, equal ones by
  ascending id, with ln p; -1 and -inf where there are no more.
  gradient of g logprob + h H:  sum over outputs of the Jacobians
    d logprob / dx_v = (1[v = t] - p_v) / T,
    d H / dx_v       = -p_v (ln p_v + H) / T.
A row left out (token -1) has logprob, H and stats 0 and no alternatives; a row
of -inf only has logprob -inf, H 0 and stats (-inf, 0); a row with NaN or
+inf has NaN everywhere and no alternatives (log probabilities NaN).

The distillation loss (App. F's masked loss with a shortened teacher row): the
teacher's entries make a distribution over the listed ids and, with a tail, one
more outcome that stands for everything else; the student's q is summed
over everything else for that outcome.  The gradient is that of the loss written
as cross-entropy with a full target: the tail's mass spread over the
unlisted ids in the student's own proportions.  The rest is 1 - sum p, taken as the largest entry's
1 - p less the others, so that it keeps its digits where one entry has nearly everything.  Only where the
student has no rest either (q_rest below 2^-100) a rest below 2^-20 is what rounding left
of a list that holds everything, and counts as none.  A teacher row that held NaN or +inf (ids -1, all log
probabilities NaN), or has NaN at an id, makes the pair's loss and gradient NaN.
"""
import numpy as np


def _log_softmax(y):
    z = y - y.max()
    return z - np.log(np.exp(z).sum())


def _plogp(logp):
    p = np.exp(logp)
    out = np.zeros_like(p)
    out[p > 0] = p[p > 0] * logp[p > 0]
    return p, out


def token_logprobs(logits, tokens=None, T=1.0, n_top=0):
    """logits [R][V] float64 values; tokens [R] or None.  Returns a dict of
    logprobs (None without tokens), entropy, stats, top_ids, top_logprobs."""
    x = np.asarray(logits, np.float64)
    R, V = x.shape
    out = dict(logprobs=None if tokens is None else np.zeros(R), entropy=np.zeros(R), stats=np.zeros((R, 2)),
               top_ids=np.full((R, n_top), -1, np.int64), top_logprobs=np.full((R, n_top), -np.inf))
    for r in range(R):
        t = 0 if tokens is None else int(tokens[r])
        if t < 0:
            continue
        if np.isnan(x[r]).any() or (x[r] == np.inf).any():
            out["entropy"][r] = out["stats"][r] = out["top_logprobs"][r] = np.nan
            if tokens is not None:
                out["logprobs"][r] = np.nan
            continue
        m = x[r].max()
        if m == -np.inf:
            out["stats"][r] = (-np.inf, 0.0)
            if tokens is not None:
                out["logprobs"][r] = -np.inf
            continue
        logp = _log_softmax(x[r] / T)
        out["stats"][r] = (m, np.log(np.exp((x[r] - m) / T).sum()))
        out["entropy"][r] = -_plogp(logp)[1].sum()
        if tokens is not None:
            out["logprobs"][r] = logp[t]
        best = sorted((v for v in range(V) if x[r, v] > -np.inf), key=lambda v: (-x[r, v], v))[:n_top]
        out["top_ids"][r, :len(best)] = best
        out["top_logprobs"][r, :len(best)] = logp[best]
    return out


def token_logprobs_grad(logits, tokens, g, h, T=1.0):
    """The gradient of sum g logprobs + h entropy; tokens, g, h [R] or None."""
    x = np.asarray(logits, np.float64)
    grad = np.zeros(x.shape)
    for r in range(x.shape[0]):
        t = 0 if tokens is None else int(tokens[r])
        if t < 0 or (x[r] == -np.inf).all():
            continue
        if np.isnan(x[r]).any() or (x[r] == np.inf).any():
            grad[r] = np.nan
            continue
        logp = _log_softmax(x[r] / T)
        p, plogp = _plogp(logp)
        if g is not None:
            grad[r] -= g[r] * p / T
            grad[r, t] = -g[r] * np.expm1(logp[t]) / T
        if h is not None:
            grad[r] -= h[r] * (plogp - p * plogp.sum()) / T
    return grad


def topk_ce(top_ids, top_logprobs, student, teacher_rows, student_rows, T=1.0, tail=True):
    """(loss, pair losses [N], gradient [R_S][V]); top_ids, top_logprobs
    [R_T][K] (id -1: no entry), student [R_S][V] float64 values."""
    x = np.asarray(student, np.float64)
    N, V = len(teacher_rows), x.shape[1]
    grad, losses = np.zeros(x.shape), np.zeros(N)
    for k, (t, s) in enumerate(zip(teacher_rows, student_rows)):
        entries = [(int(i), float(lam)) for i, lam in zip(top_ids[t], top_logprobs[t]) if i >= 0]
        ids = [i for i, _ in entries]
        assert len(set(ids)) == len(ids)
        lam_t = np.asarray(top_logprobs[t], np.float64)
        if np.isnan([lam for _, lam in entries]).any() or (not entries and np.isnan(lam_t).all()):
            losses[k] = grad[s] = np.nan
            continue
        p = np.exp(np.array([lam for _, lam in entries], np.float64))
        if not tail and p.sum() > 0:
            p = p / p.sum()
        rest = 0.0
        if tail:
            lam = np.sort(np.array([lam for _, lam in entries], np.float64))
            rest = max(0.0, -np.expm1(lam[-1]) - np.exp(lam[:-1]).sum()) if len(lam) else 1.0
        inside = np.zeros(V, bool)
        inside[ids] = True
        logq = _log_softmax(x[s] / T)
        q = np.exp(logq)
        if rest < 2.0 ** -20 and q[~inside].sum() < 2.0 ** -100:
            rest = 0.0
        if np.any(p > 0):
            i = np.array(ids)[p > 0]
            losses[k] -= (p[p > 0] * logq[i]).sum()
        target = np.zeros(V)
        target[ids] = p
        if rest > 0:
            outside = q[~inside].sum()
            losses[k] -= rest * np.log(outside)
            target[~inside] = rest * q[~inside] / outside
        grad[s] = (q * target.sum() - target) / (N * T)
    return (losses.mean() if N else 0.0), losses, grad
