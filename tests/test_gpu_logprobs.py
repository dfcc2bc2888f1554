"""Log probabilities, entropy, alternatives and their gradient on the GPU against
the float64 oracle: every element type, vocabularies from 1 to 262144 that do
and do not fill a vector, ties, masks that leave a row empty, masks of the
type's lowest value, NaN and infinities, rows left out, strided rows, the
rows used given on the device, other streams and captured calls.

Tolerances.  The kernels compute in fp32 (half a step: u = 2^-24).  With
y = (x - m) / T, each of the subtraction, the scale 1 / T and the product is off
by u, so y by 3 u |y|; its exponential by that and by the hardware's 4 u.
A sum of V exponentials over 256 threads or more adds at most V / 256 terms one
after the other and joins the threads in at most 20 steps.  Under the weights p
the mean of |y| is l - H <= ln V + (what the tail holds) < 20, so l = ln s is off by
  tol_l = u (V / 256 + 20 + 3 * 20 + 4 + 16)  (the logarithm's own rounding in the last term)
and the rest follows from the formulas by the product rule; each result is
rounded once more, by eps / 2 of its type.
"""
import math

import numpy as np
import pytest
import torch

from helpers import dev, umim
from oracle import logprobs as OL

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def tol_l(V):
    return U * (V / 256 + 100)


def f64(t):
    return t.detach().double().cpu().numpy()


def logits(seed, R, V, dtype, std=2.5, levels=None, cols=None):
    """[R][cols] with cols a multiple of 8, columns past V NaN (never to be read)."""
    cols = -(-V // 8) * 8 if cols is None else cols
    g = torch.Generator().manual_seed(seed)
    x = torch.full((R, cols), math.nan)
    x[:, :V] = std * torch.randn((R, V), generator=g)
    if levels:
        x[:, :V] = torch.round(x[:, :V] * levels) / levels
    return x.to(TYPES[dtype])


def within(got, want, tol, what):
    with np.errstate(over="ignore"):   # what leaves fp32's range is an infinity there
        got, want = np.asarray(got, np.float64), np.asarray(want).astype(np.float32).astype(np.float64)
    assert got.shape == want.shape, what
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)) and np.array_equal(np.isnan(want), np.isnan(got)), what
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
    tol = np.broadcast_to(tol, want.shape)
    over = np.abs(got[fine] - want[fine]) - tol[fine]
    assert over.size == 0 or over.max() <= 0, \
        f"{what}: {over.max():.3e} over a tolerance of {tol[fine][over.argmax()]:.3e}"


def check_forward(out, x, V, tokens=None, T=1.0, n_top=0):
    """x: what the GPU read, as a CPU tensor."""
    xd = f64(x)[:, :V]
    want = OL.token_logprobs(xd, tokens, T, n_top)
    m, l = want["stats"].T
    H = want["entropy"]
    tl = tol_l(V) + 2 * U * np.abs(np.nan_to_num(l))
    with np.errstate(invalid="ignore"):
        yt = np.abs(np.nan_to_num((xd[np.arange(len(xd)), np.maximum(tokens, 0)] - m) / T, posinf=0, neginf=0)) \
            if tokens is not None else 0.0
    if tokens is not None:
        within(f64(out["logprobs"]), want["logprobs"], tl + 5 * U * yt, "logprobs")
    spread = np.abs(np.nan_to_num(l - H))
    within(f64(out["entropy"]), H, tl + U * (V / 256 + 200) * np.maximum(1, spread), "entropy")
    within(f64(out["stats"])[:, 0], m, 0.0, "row maximum")
    within(f64(out["stats"])[:, 1], l, tl, "log of the sum")
    if n_top:
        assert np.array_equal(out["top_ids"].cpu().numpy(), want["top_ids"]), "alternatives"
        y = np.abs(np.nan_to_num(want["top_logprobs"], posinf=0, neginf=0)) + np.abs(np.nan_to_num(l))[:, None]
        within(f64(out["top_logprobs"]), want["top_logprobs"], tl[:, None] + 5 * U * y, "alternatives' values")


def check_grad(got, x, V, tokens, g, h, T, dtype):
    xd = f64(x)[:, :V]
    gd, hd = (None if g is None else f64(g)), (None if h is None else f64(h))
    want = OL.token_logprobs_grad(xd, tokens, gd, hd, T)
    o = OL.token_logprobs(xd, tokens, T)
    with np.errstate(invalid="ignore", divide="ignore"):
        z = np.nan_to_num((xd - o["stats"][:, :1]) / T - o["stats"][:, 1:], nan=0, posinf=0, neginf=-1e3)
    p, H = np.exp(z), np.abs(np.nan_to_num(o["entropy"]))[:, None]
    dp = tol_l(V) + 8 * U * (np.abs(z) + 4)     # p's own relative error
    size = p * (0 if g is None else np.abs(gd)[:, None])
    if h is not None:
        size = size + np.abs(hd)[:, None] * p * (np.abs(z) + H + 2)
    eps = torch.finfo(TYPES[dtype]).eps / 2
    tiny = 2.0 ** -25 if dtype == "fp16" else 1e-37
    # a p below 2^-126 comes out as 0, where |ln p| is below 90 if it counts at all in fp32
    tiny = tiny + 2.0 ** -126 * (np.zeros((len(xd), 1)) + (0 if g is None else np.abs(gd)[:, None])
                                 + (0 if h is None else np.abs(hd)[:, None] * (90 + H))) / T
    tol = 2 * dp * size / T + (eps + 4 * U) * np.abs(np.nan_to_num(want)) + tiny
    if h is not None:   # the entropy's own error
        tol = tol + np.abs(hd)[:, None] * p * U * (V / 256 + 300) * (1 + H) / T
    within(f64(got)[:, :V], want, tol, "gradient")


def forward(m, x, dv, V, tokens=None, T=1.0, n_top=0, **kw):
    st = m.new_status(dv)
    tok = None if tokens is None else torch.from_numpy(np.asarray(tokens, np.int32)).to(dv)
    out = m.umim_token_logprobs(x.to(dv), tok, n_top=n_top, vocab=V, temperature=T, dev_status=st, **kw)
    torch.cuda.synchronize()
    m.check_status(st)
    return out


SIZES = [  # V, R, dtype, T, n_top
    (1, 3, "bf16", 1.0, 1), (5, 4, "fp32", 0.5, 8), (7, 4, "fp16", 1.0, 3), (8, 2, "bf16", 1.0, 8),
    (33, 5, "bf16", 2.0, 33), (255, 3, "fp32", 1.0, 128), (257, 3, "fp16", 1.0, 64), (1000, 6, "bf16", 1.0, 20),
    (1001, 6, "fp32", 1.3, 5), (4096, 3, "fp16", 0.7, 128), (8191, 2, "bf16", 1.0, 17), (32000, 3, "fp32", 1.0, 128),
    (50257, 3, "bf16", 1.0, 64), (50257, 2, "fp32", 1.0, 10), (128256, 2, "bf16", 1.0, 128),
    (128256, 1, "bf16", 0.8, 20), (151936, 2, "fp16", 1.0, 20), (262144, 1, "bf16", 1.0, 128),
    (262143, 1, "fp32", 1.0, 50), (2000, 700, "bf16", 1.0, 4), (64, 3000, "fp32", 1.0, 2),
]


@pytest.mark.parametrize("V,R,dtype,T,n_top", SIZES)
def test_matches_the_oracle(V, R, dtype, T, n_top):
    m, dv = umim(), dev()
    x = logits(V + R, R, V, dtype)
    tokens = np.random.default_rng(V).integers(0, V, R)
    check_forward(forward(m, x, dv, V, tokens, T, n_top), x, V, tokens, T, n_top)


@pytest.mark.parametrize("R", [1, 2, 3, 9, 40, 151, 153, 305, 620])
def test_any_number_of_rows(R):
    """Few rows are divided among several CTAs, many are not."""
    m, dv = umim(), dev()
    V = 20011
    x = logits(R, R, V, "bf16")
    tokens = np.random.default_rng(R).integers(0, V, R)
    out = forward(m, x, dv, V, tokens, 1.0, 12)
    pick = sorted({0, R - 1, R // 2, R // 3})
    sub = {k: (v[pick] if v is not None else None) for k, v in out.items()}
    check_forward(sub, x[pick], V, tokens[pick], 1.0, 12)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("V,n_top", [(1003, 40), (40000, 128), (128256, 64)])
def test_ties_go_to_the_lowest_id(dtype, V, n_top):
    m, dv = umim(), dev()
    x = logits(3, 5, V, dtype, std=1.0, levels=1)   # whole numbers, -0 among them
    x[3, :V] = 2.0                                   # one value everywhere
    x[4, :V] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0).to(x.dtype)
    check_forward(forward(m, x, dv, V, None, 1.0, n_top), x, V, None, 1.0, n_top)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("V", [3000, 70001])
def test_sorted_rows_and_clusters_of_large_values(dtype, V):
    m, dv = umim(), dev()
    x = logits(4, 6, V, dtype)
    up = torch.linspace(-8, 8, V)
    x[0, :V], x[1, :V] = up.to(x.dtype), up.flip(0).to(x.dtype)
    x[2, V // 3:V // 3 + 200] += 20       # the best lie side by side
    x[3, V - 130:V] += 20                 # at the end
    x[4, :130] += 20                      # at the beginning
    x[5, ::max(1, V // 97)] += 20         # far apart
    for n in (1, 100, 128):
        check_forward(forward(m, x, dv, V, None, 1.0, n), x, V, None, 1.0, n)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("V", [19, 5000, 66003])
@pytest.mark.parametrize("n_top", [0, 30])
def test_masks_and_rows_without_a_distribution(dtype, V, n_top):
    m, dv = umim(), dev()
    x = logits(6, 12, V, dtype)
    low = torch.finfo(TYPES[dtype]).min
    r = np.random.default_rng(V)
    allowed = torch.from_numpy(r.choice(V, min(5, V - 1), replace=False))
    for row, fill in ((0, -math.inf), (1, low)):        # a few tokens allowed
        keep = x[row, allowed].clone()
        x[row, :V] = fill
        x[row, allowed] = keep
    x[2, :V] = -math.inf                                 # nothing allowed
    x[3, :V] = low                                       # nothing allowed, by the lowest value: uniform
    x[4, :V] = -math.inf
    x[4, V - 1] = 1.5                                    # one token allowed
    x[5, V // 2] = math.nan
    x[6, V - 1] = math.inf
    x[7, :V] = -math.inf
    x[7, V // 2] = math.nan
    x[8, : V // 2] = -math.inf                           # half of it
    x[9, :V] = -math.inf
    x[9, V // 3] = low                                   # the lowest value only
    x[10, 0] = -math.nan
    x[11, : V // 2] = low
    tokens = r.integers(0, V, 12)
    tokens[4] = V - 1
    tokens[1] = int(allowed[0])
    check_forward(forward(m, x, dv, V, tokens, 1.0, n_top), x, V, tokens, 1.0, n_top)
    check_forward(forward(m, x, dv, V, tokens, 0.05, n_top), x, V, tokens, 0.05, n_top)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_logits(dtype):
    """Values whose multiples leave fp32's range; differences that do."""
    m, dv = umim(), dev()
    V = 2049
    x = logits(8, 4, V, dtype)
    x[0, :V] = (x[0, :V].float() * 1e37).to(x.dtype)
    x[1, :V] += 2e38
    x[2, 7], x[2, 8] = 3.3e38, -3.3e38
    x[3, :V] = (x[3, :V].float() * 1e-30).to(x.dtype)
    tokens = np.array([5, 6, 7, 8])
    for T in (1.0, 1e-4, 1e4):
        check_forward(forward(m, x, dv, V, tokens, T, 9), x, V, tokens, T, 9)


def test_rows_left_out_rows_behind_the_last_and_strides():
    m, dv = umim(), dev()
    V, R = 1500, 23
    x = logits(9, R, V, "bf16", cols=1536)
    tokens = np.random.default_rng(1).integers(0, V, R)
    tokens[[0, 4, 5, 17]] = -1
    x[4] = math.nan                                     # a row left out is not read
    n = 19
    buf = x.to(dv)[:, :V]                               # a view: rows 1536 apart, vocab its columns
    st = m.new_status(dv)
    tok = torch.from_numpy(tokens.astype(np.int32)).to(dv)
    mark = dict(logprobs=torch.full((R,), 7.0, device=dv), entropy=torch.full((R,), 7.0, device=dv),
                stats=torch.full((R, 2), 7.0, device=dv),
                top_ids=torch.full((R, 6), 7, dtype=torch.int32, device=dv),
                top_logprobs=torch.full((R, 6), 7.0, device=dv))
    out = m.umim_token_logprobs(buf, tok, n_top=6, n_rows=torch.tensor([n], dtype=torch.int32, device=dv), out=mark,
                                dev_status=st)
    torch.cuda.synchronize()
    m.check_status(st)
    assert all(bool((v[n:] == 7).all()) for v in out.values())
    check_forward({k: v[:n] for k, v in out.items()}, x[:n], V, tokens[:n], 1.0, 6)
    g = torch.randn(R, device=dv)
    grad = torch.full((R, 1536), 7.0, dtype=torch.bfloat16, device=dv)
    m.umim_token_logprobs_grad(buf, out["stats"], tok, g, grad=grad, dev_status=st,
                               n_rows=torch.tensor([n], dtype=torch.int32, device=dv))
    torch.cuda.synchronize()
    m.check_status(st)
    assert bool((grad[n:] == 7).all()) and bool((grad[:, V:] == 7).all())
    check_grad(grad[:n], x[:n], V, tokens[:n], g[:n], None, 1.0, "bf16")
    for count, used in ((-3, 0), (R + 5, R)):           # clamped to [0, R]
        e = torch.full((R,), 7.0, device=dv)
        m.umim_token_logprobs(buf[:, :8], None, n_rows=torch.tensor([count], dtype=torch.int32, device=dv),
                              out=dict(entropy=e))
        torch.cuda.synchronize()
        assert int((e != 7).sum()) == used


def test_a_single_row_of_any_width():
    """One row needs no padding: its columns are all that is read."""
    m, dv = umim(), dev()
    for V, dtype in ((1, "bf16"), (50257, "bf16"), (1003, "fp32")):
        x = logits(V, 1, V, dtype)[:, :V].contiguous()
        out = m.umim_token_logprobs(x.to(dv), None, n_top=3)
        torch.cuda.synchronize()
        check_forward(out, x, V, None, 1.0, 3)
        grad = m.umim_token_logprobs_grad(x.to(dv), out["stats"], None, None, out["entropy"], torch.ones(1, device=dv))
        check_grad(grad, x, V, None, None, torch.ones(1), 1.0, dtype)


def test_bad_tokens_are_reported_and_left_out():
    m, dv = umim(), dev()
    V = 300
    x = logits(10, 4, V, "bf16")
    for bad in (V, -2, 2 ** 31 - 1, -2 ** 31):
        st = m.new_status(dv)
        tok = torch.tensor([1, bad, 2, 3], dtype=torch.int32, device=dv)
        out = m.umim_token_logprobs(x.to(dv), tok, n_top=2, vocab=V, dev_status=st)
        torch.cuda.synchronize()
        assert int(st.item()) == 1
        check_forward(out, x, V, np.array([1, -1, 2, 3]), 1.0, 2)
        st = m.new_status(dv)
        grad = m.umim_token_logprobs_grad(x.to(dv), out["stats"], tok, torch.ones(4, device=dv), vocab=V,
                                          dev_status=st)
        torch.cuda.synchronize()
        assert int(st.item()) == 1 and bool((grad[1, :V] == 0).all())


GRADS = [(V, R, dtype, T, g_on, h_on)
         for V, R, dtype, T in ((1, 2, "fp32", 1.0), (7, 3, "bf16", 1.0), (513, 4, "fp16", 0.7), (1001, 9, "fp32", 2.0),
                                (50257, 3, "bf16", 1.0), (128256, 2, "bf16", 1.0), (262144, 1, "fp32", 1.0))
         for g_on, h_on in ((True, True), (True, False), (False, True))]


@pytest.mark.parametrize("V,R,dtype,T,g_on,h_on", GRADS)
def test_gradient_matches_the_oracle(V, R, dtype, T, g_on, h_on):
    m, dv = umim(), dev()
    x = logits(V + 1, R, V, dtype)
    r = np.random.default_rng(V)
    tokens = r.integers(0, V, R)
    if R > 1:
        tokens[1] = int(x[1, :V].float().argmax())       # a likely token
        x[1, tokens[1]] += 18                            # its p so near 1 that 1 - p in fp32 would be 0
    g = torch.from_numpy(r.standard_normal(R).astype(np.float32))
    h = torch.from_numpy(r.standard_normal(R).astype(np.float32))
    out = forward(m, x, dv, V, tokens, T)
    st = m.new_status(dv)
    args = (x.to(dv), out["stats"], torch.from_numpy(tokens.astype(np.int32)).to(dv), g.to(dv) if g_on else None,
            out["entropy"], h.to(dv) if h_on else None)
    grad = m.umim_token_logprobs_grad(*args, vocab=V, temperature=T, dev_status=st)
    torch.cuda.synchronize()
    m.check_status(st)
    check_grad(grad, x, V, tokens, g if g_on else None, h if h_on else None, T, dtype)
    again = m.umim_token_logprobs_grad(*args, vocab=V, temperature=T, grad=args[0])    # in place
    assert again.data_ptr() == args[0].data_ptr() and torch.equal(again[:, :V], grad[:, :V])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_gradient_of_masked_and_bad_rows(dtype):
    m, dv = umim(), dev()
    V = 2050
    x = logits(12, 8, V, dtype)
    x[0, :V] = -math.inf
    x[1, 9] = math.nan
    x[2, 9] = math.inf
    x[3, : V - 4] = -math.inf
    x[4, : V - 4] = torch.finfo(x.dtype).min
    x[5, 3] = -math.inf
    tokens = np.array([1, 2, 3, V - 1, V - 2, 3, -1, 5])
    g, h = torch.linspace(-1, 1, 8), torch.linspace(1, 2, 8)
    out = forward(m, x, dv, V, tokens)
    tok = torch.from_numpy(tokens.astype(np.int32)).to(dv)
    grad = m.umim_token_logprobs_grad(x.to(dv), out["stats"], tok, g.to(dv), out["entropy"], h.to(dv), vocab=V)
    check_grad(grad, x, V, tokens, g, h, 1.0, dtype)


def test_gradient_is_the_difference_quotient():
    """Central differences of the GPU's own forward pass: off by d^2 / 6 times the
    third derivative (at most 2 (|g| + |h| (1 + max |ln p|)) / T^3 here) and by the two
    forward passes' errors over 2 d."""
    m, dv = umim(), dev()
    V, T, d = 37, 1.3, 2.0 ** -5
    x = logits(14, 2, V, "fp32")
    tokens = np.array([3, 30])
    tok = torch.from_numpy(tokens.astype(np.int32)).to(dv)
    g, h = torch.tensor([0.7, -1.1]), torch.tensor([0.4, 0.9])
    out = forward(m, x, dv, V, tokens, T)
    grad = f64(m.umim_token_logprobs_grad(x.to(dv), out["stats"], tok, g.to(dv), out["entropy"], h.to(dv), vocab=V,
                                          temperature=T))
    for r in range(2):
        e = torch.zeros((V, x.shape[1]))
        e[torch.arange(V), torch.arange(V)] = d
        f = []
        for sign in (1, -1):
            xs = x[r:r + 1] + sign * e
            o = m.umim_token_logprobs(xs.to(dv), tok[r:r + 1].expand(V).contiguous(), vocab=V, temperature=T)
            f.append(float(g[r]) * f64(o["logprobs"]) + float(h[r]) * f64(o["entropy"]))
        quotient = (f[0] - f[1]) / (2 * d)
        third = 2 * (abs(float(g[r])) + abs(float(h[r])) * 14) / T ** 3
        noise = 2 * (abs(float(g[r])) + abs(float(h[r]))) * (tol_l(V) * 6 + 64 * U) / (2 * d)
        within(grad[r, :V], quotient, d * d / 6 * third + noise, "difference quotient")


def test_repeatable_on_another_stream_and_from_two_at_once():
    m, dv = umim(), dev()
    V, R = 50257, 300
    x = logits(15, R, V, "bf16").to(dv)
    tok = torch.from_numpy(np.random.default_rng(2).integers(0, V, R).astype(np.int32)).to(dv)
    want = m.umim_token_logprobs(x, tok, n_top=20, vocab=V)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for s in (s1, s2):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs.append(m.umim_token_logprobs(x, tok, n_top=20, vocab=V))
    outs.append(m.umim_token_logprobs(x, tok, n_top=20, vocab=V, stream=s1))
    torch.cuda.synchronize()
    for o in outs:
        for k in want:
            assert torch.equal(o[k], want[k]), k


def test_captured_and_replayed_on_other_inputs():
    m, dv = umim(), dev()
    V, R = 4001, 9
    x = logits(16, R, V, "bf16").to(dv)
    tok = torch.zeros(R, dtype=torch.int32, device=dv)
    g, h = torch.ones(R, device=dv), torch.full((R,), 0.5, device=dv)

    def step():
        o = m.umim_token_logprobs(x, tok, n_top=7, vocab=V)
        return o, m.umim_token_logprobs_grad(x, o["stats"], tok, g, o["entropy"], h, vocab=V)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, grad = step()
    for seed in (17, 18):
        xs = logits(seed, R, V, "bf16")
        tokens = np.random.default_rng(seed).integers(0, V, R)
        x.copy_(xs)
        tok.copy_(torch.from_numpy(tokens.astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        check_forward(out, xs, V, tokens, 1.0, 7)
        check_grad(grad, xs, V, tokens, g, h, 1.0, "bf16")


def test_debug_build_gives_the_same():
    m, dv = umim(), dev()
    V, R = 30011, 5
    x = logits(19, R, V, "bf16")
    tokens = np.random.default_rng(3).integers(0, V, R)
    want = forward(m, x, dv, V, tokens, 1.0, 33)
    try:
        m.use_debug_library(True)
        got = forward(m, x, dv, V, tokens, 1.0, 33)
    finally:
        m.use_debug_library(False)
    for k in want:
        assert torch.equal(got[k], want[k]), k


def test_binding_refusals():
    m, dv = umim(), dev()
    x = torch.zeros((4, 16), dtype=torch.bfloat16, device=dv)
    tok = torch.zeros(4, dtype=torch.int32, device=dv)
    bad = [lambda: m.umim_token_logprobs(x.cpu()), lambda: m.umim_token_logprobs(x.double()),
           lambda: m.umim_token_logprobs(x.t()), lambda: m.umim_token_logprobs(x, tok.long()),
           lambda: m.umim_token_logprobs(x, tok[:3]), lambda: m.umim_token_logprobs(x, vocab=17),
           lambda: m.umim_token_logprobs(x, tok.cpu()),
           lambda: m.umim_token_logprobs_grad(x, torch.zeros((4, 2), device=dv), tok, torch.ones(4, device=dv),
                                              grad=torch.zeros((4, 24), dtype=torch.bfloat16, device=dv)),
           lambda: m.umim_token_logprobs_grad(x, torch.zeros((4, 2), device=dv), tok, torch.ones(4, device=dv),
                                              grad=x.half())]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    coded = [(1, lambda: m.umim_token_logprobs(x[:, :15].contiguous())),         # rows not 16 bytes apart
             (1, lambda: m.umim_token_logprobs(x[:, 1:9])),                      # nor on a 16-byte boundary
             (1, lambda: m.umim_token_logprobs(x, temperature=0.0)),
             (1, lambda: m.umim_token_logprobs(x, temperature=math.nan)),
             (1, lambda: m.umim_token_logprobs(x, n_top=129)),
             (1, lambda: m.umim_token_logprobs_grad(x, torch.zeros((4, 2), device=dv), tok)),
             (2, lambda: m.umim_token_logprobs(torch.zeros((1, 262145), dtype=torch.bfloat16, device=dv)))]
    for code, f in coded:
        with pytest.raises(m.UmimError) as e:
            f()
        assert e.value.code == code
    out = m.umim_token_logprobs(x[:0], tok[:0], n_top=3)     # no rows: nothing to do
    assert out["top_ids"].shape == (0, 3)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n_top", [3, 20, 128])
def test_ties_in_many_rows(dtype, n_top):
    """A CTA to each row: equal values by the hundred, and rows masked with the lowest value."""
    m, dv = umim(), dev()
    V, R = 5003, 700
    x = logits(21, R, V, dtype, std=1.5, levels=1)
    r = np.random.default_rng(5)
    low = torch.finfo(TYPES[dtype]).min
    for row in range(0, R, 7):
        keep = torch.from_numpy(r.choice(V, 9, replace=False))
        held = x[row, keep].clone()
        x[row, :V] = low if row % 2 else -math.inf
        x[row, keep] = held
    out = forward(m, x, dv, V, None, 1.0, n_top)
    ids = x[:, :V].float().sort(dim=1, descending=True, stable=True)[1][:, :n_top]
    gone = torch.gather(x[:, :V].float(), 1, ids) == -math.inf
    assert torch.equal(out["top_ids"].cpu().long(), ids.masked_fill(gone, -1))
    pick = [0, 7, 8, 350, R - 1]
    check_forward({k: (v[pick] if v is not None else None) for k, v in out.items()}, x[pick], V, None, 1.0, n_top)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("V,n_top", [(3, 3), (7, 5), (130, 128), (1999, 64), (4001, 128), (8192, 127), (16383, 128), (16385, 100)])
def test_many_alternatives_of_many_rows(dtype, V, n_top):
    """A CTA to each row, on both sides of what it reads in one go."""
    m, dv = umim(), dev()
    R = 620   # more than run at once
    x = logits(V, R, V, dtype)
    out = forward(m, x, dv, V, None, 1.0, n_top)
    ids = x[:, :V].float().sort(dim=1, descending=True, stable=True)[1][:, :n_top]
    assert torch.equal(out["top_ids"].cpu().long(), ids)
    pick = [0, 151, 152, 304, R - 1]
    check_forward({k: (v[pick] if v is not None else None) for k, v in out.items()}, x[pick], V, None, 1.0, n_top)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_value_everywhere_in_the_largest_vocabulary(dtype):
    m, dv = umim(), dev()
    V, R, n = 262144, 320, 128
    x = torch.full((R, V), -1.25, dtype=TYPES[dtype], device=dv)
    x[1::2] = torch.finfo(TYPES[dtype]).min
    out = m.umim_token_logprobs(x, n_top=n)
    torch.cuda.synchronize()
    assert torch.equal(out["top_ids"].cpu(), torch.arange(n, dtype=torch.int32).expand(R, n))
    # V equal terms: the sums of 256 threads are powers of two, so only ln rounds
    within(f64(out["entropy"]), np.full(R, math.log(V)), 16 * U * math.log(V), "entropy")


@pytest.mark.parametrize("T", [1.0, 0.01, 0.001])
@pytest.mark.parametrize("offset", [3e4, -1e5])
def test_logits_far_from_zero(T, offset):
    """x c and m c are large beside their difference: its exactness is x - m's."""
    m, dv = umim(), dev()
    V, R = 3001, 4
    x = logits(22, R, V, "fp32")
    x[:, :V] += offset
    tokens = np.array([0, 5, 2000, 3000])
    out = forward(m, x, dv, V, tokens, T, 8)
    check_forward(out, x, V, tokens, T, 8)
    g, h = torch.linspace(-1, 1, R), torch.linspace(1, 2, R)
    tok = torch.from_numpy(tokens.astype(np.int32)).to(dv)
    grad = m.umim_token_logprobs_grad(x.to(dv), out["stats"], tok, g.to(dv), out["entropy"], h.to(dv), vocab=V,
                                      temperature=T)
    check_grad(grad, x, V, tokens, g, h, T, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("V,R,n_top", [(1, 3, 1), (2, 9, 2), (700, 40, 5), (8191, 700, 0), (32000, 7, 20), (50257, 200, 0),
                                       (128256, 6, 0), (128256, 40, 3), (151936, 90, 64), (262143, 3, 10)])
def test_rows_of_one_outcome(dtype, V, R, n_top):
    """One element has nearly all of the probability: the others' share, ln s and the entropy to their own size."""
    m, dv = umim(), dev()
    T = 0.7
    r = np.random.default_rng(V + R)
    x = logits(V + R, R, V, dtype, std=1.5)
    at = np.concatenate([[0, V - 1, V // 2], r.integers(0, V, R)])[:R]
    gap = np.resize([4.0, 6.0, 10.0, 20.0, 40.0, 80.0], R)
    lse = torch.logsumexp(x[:, :V].double() / T, 1).numpy()
    x[np.arange(R), at] = torch.from_numpy(T * (lse + gap)).to(x.dtype)
    if R > 8:
        x[8, :V] = -math.inf                             # and one with nothing else
        x[8, at[8]] = 1.5
    out = forward(m, x, dv, V, at, T, n_top)
    y = f64(x)[:, :V]
    y = (y - y[np.arange(R), at][:, None]) / T
    y[np.arange(R), at] = -np.inf
    assert (y < 0).all()
    e, ay = np.exp(y), np.where(np.isinf(y), 0.0, -y)
    rest = e.sum(1)
    assert (rest < 1 / 32).all()
    H = np.log1p(rest) + (e * ay).sum(1) / (1 + rest)
    # An exponential: 3 U |y| from the exponent, 4 U its own, and from up to four changes of reference by
    # d nats 2 U |d| + 4 U each, the |d| adding up to |y| + 12; sums of V / 256 terms and less.
    # Weighed with y, a change by up to 12 loses 3 x 12 U beside terms of 3 and more.
    # Exponentials below 2^-126, where |y| is above 87.3, come out as 0: V of them at most, and as y e^-y falls
    # there, each with less than 88.4 2^-126 of entropy.
    k = U * (V / 256 + 300 + 8 * ay)
    tol_rest, tol_H = (k * e).sum(1) + V * 2.0 ** -126, (k * e * (1 + ay)).sum(1) + V * 88.4 * 2.0 ** -126
    within(f64(out["stats"])[:, 1], np.log1p(rest), tol_rest, "log of the sum")
    within(f64(out["logprobs"]), -np.log1p(rest), tol_rest, "logprobs")
    within(f64(out["entropy"]), H, tol_H, "entropy")
    if n_top:
        assert np.array_equal(out["top_ids"][:, 0].cpu().numpy(), at)
        within(f64(out["top_logprobs"])[:, 0], -np.log1p(rest), tol_rest, "best alternative")
    # two of them share it: neither is certain
    other = (at + 1) % V
    x[np.arange(R), other] = x[np.arange(R), at]
    out = forward(m, x, dv, V, at, T, n_top)
    few = slice(0, 10)
    check_forward({k: (v[few] if v is not None else None) for k, v in out.items()}, x[few], V, at[few], T, n_top)


def test_rows_beyond_32_bits_of_elements():
    m, dv = umim(), dev()
    V, R = 128256, 17000                                  # 2.18e9 elements; only the first and last rows count
    x = torch.empty((R, V), dtype=torch.bfloat16, device=dv)
    some = [0, R - 2, R - 1]
    part = logits(31, 3, V, "bf16")
    x[some] = part.to(dv)
    tokens = np.full(R, -1, np.int32)
    tokens[some] = [5, 128255, 77]
    tok = torch.from_numpy(tokens).to(dv)
    out = m.umim_token_logprobs(x, tok, n_top=9)
    sub = {k: v[some] for k, v in out.items()}
    check_forward(sub, part, V, tokens[some], 1.0, 9)
    g = torch.ones(R, device=dv)
    grad = m.umim_token_logprobs_grad(x, out["stats"], tok, g, grad=x)
    torch.cuda.synchronize()
    check_grad(grad[some], part, V, tokens[some], g[some], None, 1.0, "bf16")
    assert not bool(grad[1].any()) and not bool(grad[R - 3].any())
