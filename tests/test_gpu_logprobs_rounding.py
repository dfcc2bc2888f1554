"""Log probabilities far below 0 are rounded once, whatever the temperature.

With bf16 logits of few exponents x - m is exact.  (x - m) / T takes both parts of 1 / T, whose product is left unrounded
by FMA, so what remains is half a step of the result, u = 2^-24 of it, beside ln s's own error tol_l.  Temperatures are
those whose reciprocal fp32 rounds worst: rounding it, the product and the difference cost 3 u.
"""
import numpy as np
import pytest
import torch

from helpers import dev, umim
from oracle import logprobs as OL
from test_gpu_logprobs import U, f64, logits, tol_l, within

pytestmark = pytest.mark.gpu


def worst_temperatures(lo, hi, n):
    """fp32 temperatures in [lo, hi] whose fp32 reciprocals are off by the most."""
    t = np.random.default_rng(1).uniform(lo, hi, 4000).astype(np.float32).astype(np.float64)
    off = np.abs((1 / t).astype(np.float32).astype(np.float64) * t - 1)
    return t[np.argsort(-off)[:n]]


@pytest.mark.parametrize("n_top", [0, 30])
@pytest.mark.parametrize("T", worst_temperatures(0.006, 0.02, 3).tolist() + worst_temperatures(0.5, 2.0, 2).tolist())
def test_one_rounding(T, n_top):
    m, dv = umim(), dev()
    V, R = 64, 200
    x = logits(3, R, V, "bf16")
    tokens = np.random.default_rng(2).integers(0, V, R)
    st = m.new_status(dv)
    out = m.umim_token_logprobs(x.to(dv), torch.from_numpy(tokens.astype(np.int32)).to(dv), n_top=n_top, vocab=V,
                                temperature=T, dev_status=st)
    torch.cuda.synchronize()
    m.check_status(st)
    want = OL.token_logprobs(f64(x)[:, :V], tokens, float(np.float32(T)), n_top)
    tol = lambda v: 1.05 * U * np.abs(v) + tol_l(V)
    within(f64(out["logprobs"]), want["logprobs"], tol(want["logprobs"]), "log probabilities")
    if n_top:
        within(f64(out["top_logprobs"]), want["top_logprobs"], tol(want["top_logprobs"]), "alternatives")
