"""Distillation from the teacher's top log probabilities on the GPU against the
float64 oracle: loss, pair losses and gradient with and without the tail, every
element type, lists of 1 to 128 ids, vocabularies from 1 to 262144, masked and
bad rows, pairs given on the device, and the whole path from the teacher's
logits through the cache to the student's gradient.

Tolerances: those of test_gpu_logprobs.py (u = 2^-24, tol_l the error of the
log of a sum over the vocabulary).  A pair's loss sums p_i ln q_i, each p_i off
by 8 u (its exponential and the sum it is divided by), each ln q_i by
tol_l + 8 u |y_i|; the rest is one minus a sum of K terms, off by (K + 8) u.  The gradient's
factor P - p_rest / q_rest is off by both parts' errors, and is rounded once by
eps / 2 of its type.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import workloads as W
from helpers import dev, umim
from oracle import distill as OD
from oracle import logprobs as OL
from test_gpu_logprobs import TYPES, U, f64, logits, tol_l, within

pytestmark = pytest.mark.gpu


def lists(seed, R_T, K, V, holes=True, mass=0.9):
    """[R_T][K] distinct ids in random places, log probabilities that sum to `mass`."""
    r = np.random.default_rng(seed)
    K_held = min(K, V)
    if K_held == V:
        mass = 1.0     # the whole vocabulary: nothing is left
    ids = np.full((R_T, K), -1, np.int32)
    lp = np.full((R_T, K), -np.inf, np.float32)
    for t in range(R_T):
        at = r.permutation(K)[:K_held] if holes and t % 3 == 2 else np.arange(K_held)
        ids[t, at] = r.choice(V, K_held, replace=False)
        w = np.exp(2.0 * r.standard_normal(K_held))
        lp[t, at] = np.log(mass * w / w.sum())
    return ids, lp


def near(x, ids, lp, tr, sr, T):
    """Student rows raised at the teacher's ids, as a student that has learned something."""
    for t, s in zip(tr, sr):
        held = ids[t] >= 0
        if held.any():
            x[s, torch.from_numpy(ids[t][held]).long()] = \
                torch.from_numpy(T * (np.maximum(lp[t][held], -30) + 9.0)).to(x.dtype)
    return x


def run(m, dv, ids, lp, x, V, tr, sr, T=1.0, tail=True, expect=0, **kw):
    st = m.new_status(dv)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).to(dv)
    values = torch.from_numpy(np.ascontiguousarray(np.asarray(lp, np.float32))).to(dv)
    out = m.umim_distill_topk_ce(i32(ids), values, x.to(dv), i32(tr), i32(sr), vocab=V, temperature=T, tail=tail,
                                 dev_status=st, **kw)
    torch.cuda.synchronize()
    assert int(st.item()) == expect
    return out


def check(out, ids, lp, x, V, tr, sr, T, tail, dtype, scale=1.0):
    loss, pair_loss, grad = out
    xd = f64(x)[:, :V]
    N, K = len(tr), ids.shape[1]
    want, pairs, wgrad = OL.topk_ce(ids, lp, xd, tr, sr, T, tail)
    tols = np.zeros(N)
    gtol = np.zeros((len(xd), V))
    eps = torch.finfo(TYPES[dtype]).eps / 2
    for k, (t, s) in enumerate(zip(tr, sr)):
        with np.errstate(all="ignore"):
            logq = OL._log_softmax(xd[s] / T)
        held = ids[t] >= 0
        p = np.exp(lp[t][held].astype(np.float64))
        p = p / p.sum() if not tail and p.sum() > 0 else p
        rest = max(0.0, 1 - p.sum()) if tail else 0.0
        inside = np.zeros(V, bool)
        inside[ids[t][held]] = True
        q = np.exp(np.nan_to_num(logq, nan=0, neginf=-1e3, posinf=0))
        q_rest = max(q[~inside].sum(), 1e-300)
        y = np.abs(np.nan_to_num(logq[ids[t][held]], nan=0, neginf=0, posinf=0)) + 20
        e = tol_l(V) + 8 * U * (y.max() if held.any() else 1)
        tols[k] = 2 * e + U * (K + 8) * ((y.max() if held.any() else 1) + abs(math.log(q_rest)) * (rest > 0))
        d = 4 * (tol_l(V) + 8 * U * (np.abs(np.nan_to_num(logq, nan=0, neginf=-100, posinf=0)) + 24))
        row = q * (1 + rest / q_rest) * d + (q * U * (K + 8) / q_rest if rest > 0 else 0)
        row[ids[t][held]] = (q[ids[t][held]] + p) * (d[ids[t][held]] + U * (K + 8))
        gtol[s] = abs(scale) * row / (N * T)
    within(f64(pair_loss)[:N], pairs, tols, "pair losses")
    within(f64(loss), [want], (tols.mean() if N else 0) + 4 * U * abs(np.nan_to_num(want)), "loss")
    if grad is not None:
        wgrad = wgrad * scale
        tiny = 2.0 ** -25 if dtype == "fp16" else 1e-37
        # an exponential below 2^-126 comes out as 0; what it is multiplied by is at most P + p_rest <= 2 over N T
        tiny += 2.0 ** -126 * 2 * abs(scale) / (max(N, 1) * T)
        within(f64(grad)[:, :V], wgrad, gtol + (eps + 4 * U) * np.abs(np.nan_to_num(wgrad)) + tiny, "gradient")


CASES = [  # V, R_T, R_S, N, K, dtype, T
    (1, 2, 2, 2, 1, "fp32", 1.0), (5, 3, 4, 3, 8, "bf16", 1.0), (9, 2, 3, 2, 4, "fp16", 0.5),
    (64, 5, 9, 6, 64, "fp32", 1.0), (500, 20, 30, 25, 128, "bf16", 1.0), (1001, 9, 11, 7, 20, "fp32", 2.0),
    (4096, 4, 6, 4, 1, "bf16", 1.0),
    (8195, 4, 5, 3, 33, "fp16", 1.0), (32000, 3, 4, 3, 50, "bf16", 0.7), (50257, 3, 3, 2, 128, "fp32", 1.0),
    (128256, 3, 3, 2, 64, "bf16", 1.0), (151936, 2, 2, 2, 100, "fp16", 1.0), (262144, 2, 2, 1, 128, "bf16", 1.0),
    (262143, 1, 1, 1, 20, "fp32", 1.0), (1500, 50, 800, 650, 10, "bf16", 1.0),
]


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("V,R_T,R_S,N,K,dtype,T", CASES)
def test_matches_the_oracle(V, R_T, R_S, N, K, dtype, T, tail):
    m, dv = umim(), dev()
    r = np.random.default_rng(V + K)
    ids, lp = lists(V, R_T, K, V)
    tr = r.integers(0, R_T, N)               # a teacher row may serve several pairs
    sr = np.sort(r.permutation(R_S)[:N])
    x = near(logits(V, R_S, V, dtype), ids, lp, tr, sr, T)
    out = run(m, dv, ids, lp, x, V, tr, sr, T, tail)
    check(out, ids, lp, x, V, tr, sr, T, tail, dtype)
    unpaired = np.setdiff1d(np.arange(R_S), sr)
    assert bool((out[2][torch.from_numpy(unpaired).to(dv)][:, :V] == 0).all())


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("R_S", [1, 2, 5, 17, 80, 160, 310])
def test_any_number_of_rows(R_S, tail):
    m, dv = umim(), dev()
    V, K = 20011, 40
    r = np.random.default_rng(R_S)
    N = max(1, R_S * 3 // 4)
    ids, lp = lists(R_S, N, K, V)
    tr, sr = r.permutation(N), r.permutation(R_S)[:N]
    x = near(logits(R_S, R_S, V, "bf16"), ids, lp, tr, sr, 1.0)
    check(run(m, dv, ids, lp, x, V, tr, sr, 1.0, tail), ids, lp, x, V, tr, sr, 1.0, tail, "bf16")


def test_full_lists_give_the_full_vocabulary_loss():
    """Every id listed: App. F's soft cross-entropy over the whole vocabulary, by
    the library's own full-vocabulary call too."""
    m, dv = umim(), dev()
    V, R = 120, 12
    teacher, x = logits(1, R, V, "bf16"), logits(2, R, V, "bf16")
    st = m.new_status(dv)
    cache = m.umim_token_logprobs(teacher.to(dv), n_top=V, vocab=V, dev_status=st)
    tr, sr = np.arange(R)[::-1].copy(), np.arange(R)
    i32 = lambda a: torch.from_numpy(a.astype(np.int32)).to(dv)
    full = m.umim_distill_soft_ce(teacher.to(dv), x.to(dv), i32(tr), i32(sr), vocab=V, eps=0.0, dev_status=st)
    want, wgrad = OD.soft_ce(f64(teacher)[:, :V], f64(x)[:, :V], tr, sr, eps=0.0)
    for tail in (True, False):
        loss, pairs, grad = m.umim_distill_topk_ce(cache["top_ids"], cache["top_logprobs"], x.to(dv), i32(tr), i32(sr),
                                                   vocab=V, tail=tail, dev_status=st)
        torch.cuda.synchronize()
        m.check_status(st)
        assert abs(loss.item() - want) < 1e-5 * want and abs(loss.item() - full[0].item()) < 1e-5 * want
        # 16 roundings of P q - p with both parts below 1 / R, and the output's own
        within(f64(grad)[:, :V], wgrad, 200 * U / R + 2.0 ** -8 * np.abs(wgrad), "gradient")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("V", [600, 33001])
def test_masked_and_bad_student_rows(dtype, tail, V):
    m, dv = umim(), dev()
    K, R = 16, 8
    ids, lp = lists(5, R, K, V, holes=False)
    lp[5, 3:] = -np.inf                                  # entries of no probability
    ids[6] = -1                                          # a teacher row without entries
    tr = sr = np.arange(R)
    x = near(logits(5, R, V, dtype), ids, lp, tr, sr, 1.0)
    outside = np.ones(V, bool)
    outside[ids[0]] = False
    x[0, torch.from_numpy(np.nonzero(outside)[0][5:])] = -math.inf      # most of the rest masked
    x[1, torch.from_numpy(np.setdiff1d(np.arange(V), ids[1])[5:])] = torch.finfo(x.dtype).min
    x[5, torch.from_numpy(ids[5, 3:]).long()] = -math.inf               # masked where nothing is asked
    x[2, :V] = -math.inf
    x[3, V - 1] = math.nan
    x[4, V - 2] = math.inf
    loss, pairs, grad = run(m, dv, ids, lp, x, V, tr, sr, 1.0, tail)
    good = [0, 1, 5, 6, 7]
    got = torch.stack([pairs[k] for k in good])
    n = len(good)
    g = grad[good]
    check((got.double().mean().reshape(1), got, g), ids[good], lp[good], x[good], V, np.arange(n), np.arange(n), 1.0,
          tail, dtype, scale=n / R)
    assert pairs[2].item() == math.inf and bool((grad[2, :V] == 0).all())
    for k in (3, 4):
        assert math.isnan(pairs[k].item()) and bool(grad[k, :V].isnan().all())
    assert math.isnan(loss.item())
    # what is masked in the student and asked for by the teacher costs infinitely much; its gradient is finite
    x = logits(6, 1, V, dtype)
    x[0, int(ids[0, 0])] = -math.inf
    loss, pairs, grad = run(m, dv, ids, lp, x, V, [0], [0], 1.0, tail)
    assert pairs[0].item() == math.inf and bool(torch.isfinite(grad[:, :V]).all())


def test_a_list_that_holds_all_there_is():
    """Teacher and student under the same mask, the list complete: the log
    probabilities' rounding leaves no rest to be looked for where q_rest is 0."""
    m, dv = umim(), dev()
    V, K = 5000, 24
    r = np.random.default_rng(4)
    allowed = r.permutation(V)[:20]
    t, x = logits(1, 3, V, "bf16"), logits(2, 3, V, "bf16")
    blocked = torch.from_numpy(np.setdiff1d(np.arange(V), allowed))
    t[:, blocked] = -math.inf
    x[:, blocked] = -math.inf
    c = m.umim_token_logprobs(t.to(dv), n_top=K, vocab=V)
    ids, lp = c["top_ids"].cpu().numpy(), c["top_logprobs"].cpu().numpy()
    assert (ids[:, 20:] == -1).all() and (ids[:, :20] >= 0).all()
    tr = sr = np.arange(3)
    out = run(m, dv, ids, lp, x, V, tr, sr)
    assert bool(torch.isfinite(out[0]).all()) and bool(torch.isfinite(out[2][:, :V]).all())
    check(out, ids, lp, x, V, tr, sr, 1.0, True, "bf16")


def test_scale_loss_only_padding_pairs_on_the_device_and_no_pairs():
    m, dv = umim(), dev()
    V, K, R = 1001, 9, 20
    ids, lp = lists(7, R, K, V)
    r = np.random.default_rng(7)
    tr, sr = r.permutation(R), r.permutation(R)
    x = near(logits(7, R, V, "bf16", cols=1016), ids, lp, tr, sr, 1.0)
    g = torch.full((R, 1016), 9.0, dtype=torch.bfloat16, device=dv)
    a = run(m, dv, ids, lp, x, V, tr, sr, grad_scale=-64.0, grad=g)
    assert bool((g[:, V:] == 9).all())
    check(a, ids, lp, x, V, tr, sr, 1.0, True, "bf16", scale=-64.0)
    b = run(m, dv, ids, lp, x, V, tr, sr, with_grad=False)
    assert b[2] is None and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    n = 13
    pairs = torch.full((R,), 5.0, device=dv)
    c = run(m, dv, ids, lp, x, V, tr, sr, n_pairs=torch.tensor([n], dtype=torch.int32, device=dv), pair_loss=pairs)
    assert bool((pairs[n:] == 5).all())
    check(c, ids, lp, x, V, tr[:n], sr[:n], 1.0, True, "bf16")
    d = run(m, dv, ids, lp, x, V, [], [])
    assert d[0].item() == 0 and bool((d[2][:, :V] == 0).all())
    e = run(m, dv, ids, lp, x[:0], V, [], [])
    assert e[0].item() == 0 and e[2].shape[0] == 0
    f = run(m, dv, ids[:0], lp[:0], x, V, [], [])
    assert f[0].item() == 0


def test_invalid_pairs_write_nothing():
    m, dv = umim(), dev()
    V, K, R = 640, 5, 8
    ids, lp = lists(8, R, K, V)
    x = logits(8, R, V, "bf16")
    base = np.arange(R)
    for what in ("twice", "teacher", "student", "negative", "count", "count below 0"):
        tr, sr, n = base.copy(), base.copy(), None
        if what == "twice":
            sr[3] = sr[5]
        elif what == "teacher":
            tr[1] = R
        elif what == "student":
            sr[7] = R
        elif what == "negative":
            tr[0] = -1
        else:
            n = torch.tensor([R + 1 if what == "count" else -1], dtype=torch.int32, device=dv)
        g, lo = torch.full_like(x, 3.0).to(dv), torch.full((1,), 5.0, device=dv)
        pl = torch.full((R,), 6.0, device=dv)
        run(m, dv, ids, lp, x, V, tr, sr, expect=1, n_pairs=n, grad=g, loss=lo, pair_loss=pl)
        assert bool((g == 3).all()) and lo.item() == 5 and bool((pl == 6).all()), what


def test_bad_ids_are_reported_and_count_as_none():
    m, dv = umim(), dev()
    V, K, R = 640, 12, 4
    ids, lp = lists(9, R, K, V, holes=False)
    x = logits(9, R, V, "bf16")
    tr = sr = np.arange(R)
    for bad in (V, -2, 2 ** 31 - 1, -2 ** 31, "twice"):
        b, want = ids.copy(), ids.copy()
        b[2, 7] = ids[2, 3] if bad == "twice" else bad
        want[2, 7] = -1
        for tail in (True, False):
            check(run(m, dv, b, lp, x, V, tr, sr, 1.0, tail, expect=1), want, lp, x, V, tr, sr, 1.0, tail, "bf16")


def test_repeatable_captured_and_on_another_stream():
    m, dv = umim(), dev()
    V, K, R = 30001, 50, 40
    ids, lp = lists(10, R, K, V)
    tr = sr = np.arange(R)
    x = near(logits(10, R, V, "bf16"), ids, lp, tr, sr, 1.0)
    a = run(m, dv, ids, lp, x, V, tr, sr)
    b = run(m, dv, ids, lp, x, V, tr, sr)
    with torch.cuda.stream(torch.cuda.Stream()):
        c = run(m, dv, ids, lp, x, V, tr, sr)
    for o in (b, c):
        assert torch.equal(a[0], o[0]) and torch.equal(a[1], o[1]) and torch.equal(a[2][:, :V], o[2][:, :V])
    i32 = lambda v: torch.from_numpy(np.asarray(v, np.int32)).to(dv)
    bufs = dict(ids=i32(ids), lp=torch.from_numpy(lp).to(dv), x=x.to(dv), tr=i32(tr), sr=i32(sr))
    ws = m.workspace(m.umim_distill_topk_ce_workspace_size(R, R), dv)
    ws.fill_(0xA5)                                        # its contents do not matter
    step = lambda: m.umim_distill_topk_ce(bufs["ids"], bufs["lp"], bufs["x"], bufs["tr"], bufs["sr"], vocab=V,
                                          workspace_buf=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (11, 12):
        ids, lp = lists(seed, R, K, V)
        sr = np.random.default_rng(seed).permutation(R)
        x = near(logits(seed, R, V, "bf16"), ids, lp, tr, sr, 1.0)
        for name, v in (("ids", i32(ids)), ("lp", torch.from_numpy(lp)), ("x", x), ("sr", i32(sr))):
            bufs[name].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        check(out, ids, lp, x, V, tr, sr, 1.0, True, "bf16")


def test_debug_build_gives_the_same():
    m, dv = umim(), dev()
    V, K, R = 9000, 30, 6
    ids, lp = lists(13, R, K, V)
    tr = sr = np.arange(R)
    x = near(logits(13, R, V, "fp16"), ids, lp, tr, sr, 1.0)
    a = run(m, dv, ids, lp, x, V, tr, sr)
    try:
        m.use_debug_library(True)
        b = run(m, dv, ids, lp, x, V, tr, sr)
    finally:
        m.use_debug_library(False)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2][:, :V], b[2][:, :V])


def test_gradient_is_the_difference_quotient():
    """Central differences of the GPU's own loss, one student row per shifted
    element: off by d^2 / 6 times the third derivative (at most 2 / T^3 for weights that sum to 1, twice
    for the two logarithms) and the pair losses' errors over 2 d."""
    m, dv = umim(), dev()
    V, K, T, d = 41, 6, 1.2, 2.0 ** -5
    ids, lp = lists(14, 1, K, V)
    x = near(logits(14, 1, V, "fp32"), ids, lp, [0], [0], T)
    grad = f64(run(m, dv, ids, lp, x, V, [0], [0], T)[2])[0, :V]
    e = torch.zeros((V, x.shape[1]))
    e[torch.arange(V), torch.arange(V)] = d
    f = [f64(run(m, dv, ids, lp, x + s * e, V, np.zeros(V), np.arange(V), T, with_grad=False)[1]) for s in (1, -1)]
    noise = 2 * (3 * tol_l(V) + 400 * U) / (2 * d)
    within(grad, (f[0] - f[1]) / (2 * d), d * d / 6 * 4 / T ** 3 + noise, "difference quotient")


@pytest.mark.parametrize("V,lens", [(1003, [40, 0, 75, 23, 9]), (32000, [64, 31])])
def test_the_whole_path_from_the_teacher_to_the_students_gradient(V, lens):
    """A training step's calls: the teacher's cache, the alignment, the
    distillation loss, hard labels and an entropy term on the aligned rows, the
    two gradients added; the student's perplexity from the same call."""
    m, dv = umim(), dev()
    K, T = 20, 1.5
    c = W.distill_case(71 + V, lens=lens, vocab=V, coverage=0.4, device=dv)
    offs, tp, sp = OD.align(np.array(lens), *(t.cpu().numpy() for t in (c.span_offsets, c.span_start, c.span_len)))
    so, sl = c.span_offsets.cpu().numpy(), c.span_len.cpu().numpy()
    L_c = np.array([lens[b] - int((sl[so[b]:so[b + 1]] - 1).sum()) for b in range(len(lens))])
    which = np.repeat(np.arange(len(lens)), np.diff(offs))
    tr = np.concatenate([[0], np.cumsum(lens)])[which] + tp
    sr = np.concatenate([[0], np.cumsum(L_c)])[which] + sp
    R_S, N = int(L_c.sum()), len(tr)
    student = W.distill_logits(72 + V, R_S, c.teacher_logits.shape[1], 2.0, dv)
    st = m.new_status(dv)
    cache = m.umim_token_logprobs(c.teacher_logits, n_top=K, vocab=V, temperature=T, dev_status=st)
    al = m.umim_distill_align(c.seq_lens, c.span_offsets, c.span_start, c.span_len, int(sum(lens)), dev_status=st)
    loss, pairs, grad = m.umim_distill_topk_ce(cache["top_ids"], cache["top_logprobs"], student, al["teacher_rows"],
                                               al["student_rows"], n_pairs=al["pair_offsets"][-1:], vocab=V,
                                               temperature=T, grad_scale=T * T, dev_status=st)
    labels = np.full(R_S, -1, np.int32)
    labels[sr] = np.random.default_rng(V).integers(0, V, N)
    tok = torch.from_numpy(labels).to(dv)
    fwd = m.umim_token_logprobs(student, tok, vocab=V, dev_status=st)
    g = torch.full((R_S,), -0.5 / N, device=dv)
    h = torch.full((R_S,), 0.1 / N, device=dv)
    g2 = m.umim_token_logprobs_grad(student, fwd["stats"], tok, g, fwd["entropy"], h, vocab=V, dev_status=st)
    total = grad[:, :V].float() + g2[:, :V].float()
    torch.cuda.synchronize()
    m.check_status(st)
    xd, td = f64(student)[:, :V], f64(c.teacher_logits)[:, :V]
    o = OL.token_logprobs(td, None, T, K)
    assert np.array_equal(cache["top_ids"].cpu().numpy(), o["top_ids"])
    want, _, wgrad = OL.topk_ce(o["top_ids"], o["top_logprobs"], xd, tr, sr, T, True)
    w2 = OL.token_logprobs_grad(xd, labels, f64(g), f64(h), 1.0)
    assert abs(loss.item() - want) <= 1e-5 * want          # 1e-5 = 168 u: tol_l and the cache's own
    ppl = OL.token_logprobs(xd, labels)["logprobs"][labels >= 0].mean()
    assert abs(fwd["logprobs"][tok >= 0].double().mean().item() - ppl) <= 1e-5 * abs(ppl)
    # two bf16 roundings (2^-9 each, relative to their own value) and the fp32 errors of values below 2 / N
    tol = 2.0 ** -8 * (np.abs(wgrad * T * T) + np.abs(w2)) + 3000 * U / N
    within(f64(total), wgrad * T * T + w2, tol, "the step's gradient")
    assert oracle.logprobs is OL


def test_binding_refusals():
    m, dv = umim(), dev()
    ids = torch.zeros((2, 3), dtype=torch.int32, device=dv)
    lp = torch.zeros((2, 3), device=dv)
    x = torch.zeros((2, 16), dtype=torch.bfloat16, device=dv)
    rows = torch.arange(2, dtype=torch.int32, device=dv)
    bad = [lambda: m.umim_distill_topk_ce(ids.long(), lp, x, rows, rows),
           lambda: m.umim_distill_topk_ce(ids, lp.half(), x, rows, rows),
           lambda: m.umim_distill_topk_ce(ids, lp[:, :2], x, rows, rows),
           lambda: m.umim_distill_topk_ce(ids, lp, x.double(), rows, rows),
           lambda: m.umim_distill_topk_ce(ids, lp, x, rows.long(), rows),
           lambda: m.umim_distill_topk_ce(ids, lp, x, rows, rows[:1]),
           lambda: m.umim_distill_topk_ce(ids, lp, x, rows, rows, vocab=17),
           lambda: m.umim_distill_topk_ce(ids, lp, x, rows, rows, grad=x.float())]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    wide = torch.zeros((2, 129), dtype=torch.int32, device=dv)
    coded = [(1, lambda: m.umim_distill_topk_ce(wide, wide.float(), x, rows, rows)),
             (1, lambda: m.umim_distill_topk_ce(ids[:, :0].contiguous(), lp[:, :0].contiguous(), x, rows, rows)),
             (1, lambda: m.umim_distill_topk_ce(ids, lp, x, rows, rows, temperature=-1.0)),
             (1, lambda: m.umim_distill_topk_ce(ids, lp, x, rows, rows, grad_scale=math.inf)),
             (5, lambda: m.umim_distill_topk_ce(ids, lp, x, rows, rows, workspace_buf=m.workspace(256, dv)))]
    for code, f in coded:
        with pytest.raises(m.UmimError) as e:
            f()
        assert e.value.code == code


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("T", [1.0, 0.01, 0.001])
@pytest.mark.parametrize("offset", [3e4, -1e5])
def test_logits_far_from_zero(offset, T, tail):
    """x c and m c are large beside their difference: its exactness is x - m's."""
    m, dv = umim(), dev()
    V, K, R = 3001, 20, 5
    ids, lp = lists(15, R, K, V)
    tr = sr = np.arange(R)
    x = logits(15, R, V, "fp32")
    x[:, :V] += offset
    check(run(m, dv, ids, lp, x, V, tr, sr, T, tail), ids, lp, x, V, tr, sr, T, tail, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V,R,N", [(12000, 600, 513), (70000, 400, 399), (300, 2000, 1999),
                                   # clusters of 3, 5, 6 and 7 for bf16, of 6 and 7 for fp32
                                   (96001, 330, 310), (151936, 200, 190), (185003, 170, 160), (215001, 130, 121)])
def test_more_pairs_than_clusters(dtype, V, R, N):
    """Clusters take pair after pair: every row of the gradient against plain torch in float64."""
    m, dv = umim(), dev()
    K, T = 30, 1.2
    r = np.random.default_rng(V)
    ids, lp = lists(16, 50, K, V, holes=False)
    tr, sr = r.integers(0, 50, N), r.permutation(R)[:N]
    x = logits(16, R, V, dtype)
    loss, pairs, grad = run(m, dv, ids, lp, x, V, tr, sr, T, True)
    s, t = torch.from_numpy(sr).to(dv), torch.from_numpy(tr).to(dv)
    logq = torch.log_softmax(x.to(dv)[s, :V].double() / T, 1)
    at = torch.from_numpy(ids).to(dv).long()[t]
    p = torch.from_numpy(lp).to(dv).double()[t].exp()
    rest = 1 - p.sum(1)
    q_rest = logq.exp().scatter(1, at, 0.0).sum(1)
    want = -(p * logq.gather(1, at)).sum(1) - rest * q_rest.log()
    # every |ln q| here is below 40, p sums to 1
    tol = 2 * tol_l(V) + U * (8 + K + 8) * 40
    within(f64(pairs), want.cpu().numpy(), tol, "pair losses")
    within(f64(loss), [want.mean().item()], tol, "loss")
    d = logq.exp() * (1 - rest / q_rest)[:, None]
    d.scatter_(1, at, logq.exp().gather(1, at) * 1.0 - p)
    wgrad = torch.zeros((R, V), dtype=torch.float64, device=dv)
    wgrad[s] = d / (N * T)
    size = torch.zeros((R, V), dtype=torch.float64, device=dv)
    size[s] = logq.exp() * (1 + rest / q_rest)[:, None] + torch.zeros_like(logq).scatter(1, at, p)
    eps = torch.finfo(TYPES[dtype]).eps / 2
    factor = 4 * (tol_l(V) + 8 * U * 64 + U * (K + 8)) / (N * T)
    off = (grad[:, :V].double() - wgrad).abs() - (eps + 4 * U) * wgrad.abs() - factor * size
    assert bool((off <= 1e-37).all())


def test_rows_beyond_32_bits_of_elements():
    m, dv = umim(), dev()
    V, R, K = 128256, 17000, 10                           # 2.18e9 elements; only the first and last rows are paired
    x = torch.empty((R, V), dtype=torch.bfloat16, device=dv)
    ids, lp = lists(33, 3, K, V)
    part = near(logits(33, 3, V, "bf16"), ids, lp, range(3), range(3), 1.0)
    sr = np.array([R - 1, 0, R - 2])
    x[torch.from_numpy(sr).to(dv)] = part.to(dv)
    i32 = lambda a: torch.from_numpy(np.asarray(a, np.int32)).to(dv)
    st = m.new_status(dv)
    loss, pairs, grad = m.umim_distill_topk_ce(i32(ids), torch.from_numpy(lp).to(dv), x, i32(np.arange(3)), i32(sr),
                                               dev_status=st)
    torch.cuda.synchronize()
    m.check_status(st)
    same = np.arange(3)
    check((loss, pairs, grad[torch.from_numpy(sr).to(dv)]), ids, lp, part, V, same, same, 1.0, True, "bf16")
    assert not bool(grad[1:R - 2].any())
