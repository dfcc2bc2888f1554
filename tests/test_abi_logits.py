"""Host-side checks of the calls over rows of logits (log probabilities, their
gradient, distillation from top log probabilities), without a GPU: every call
below stops at a check, before the first CUDA call."""
import ctypes
import math
import os

import pytest


@pytest.fixture(scope="module", params=["release", "debug"])
def lib(request):
    from paper_2609_27233_gb300 import build, _lib
    path = _lib.LIB_PATH if request.param == "release" else _lib.DEBUG_LIB_PATH
    if not os.path.exists(path):
        build.build(variants=(request.param,))
    return _lib.load(path)


null = ctypes.c_void_p(0)
fake = ctypes.c_void_p(1 << 20)      # never dereferenced
odd = ctypes.c_void_p((1 << 20) + 4)
nan = math.nan


def test_token_logprobs(lib):
    def call(x=fake, dtype=0, R=4, V=1000, ld=1000, tok=fake, T=1.0, n=0, lp=fake, stats=fake, ids=null, tl=null):
        return lib.umim_token_logprobs(x, dtype, R, V, ld, null, tok, T, n, lp, fake, stats, ids, tl, null, null)
    assert call(x=null) == 1
    assert call(x=odd) == 1                       # not 16-byte aligned
    assert call(dtype=3) == 1 and call(dtype=-1) == 1
    assert call(R=-1) == 1 and call(V=0) == 1
    assert call(V=1001, ld=1001) == 1             # rows not 16 bytes apart
    assert call(dtype=2, V=1002, ld=1002) == 1
    assert call(V=1000, ld=992) == 1              # rows overlap
    assert call(V=262145, ld=262152) == 2         # vocabulary above the largest
    assert call(R=2 ** 30 + 1) == 2               # and rows
    for T in (0.0, -1.0, nan, math.inf, 1e-5, 1e5):
        assert call(T=T) == 1, T
    assert call(n=-1) == 1 and call(n=129) == 1
    assert call(n=5) == 1                         # alternatives without arrays for them
    assert call(n=5, ids=fake) == 1
    assert call(tok=null) == 1                    # log probabilities of no tokens
    assert call(stats=odd) == 1
    assert call(R=0) == 0 and call(R=0, x=null) == 0


def test_token_logprobs_grad(lib):
    def call(x=fake, dtype=0, R=4, V=1000, ld=1000, tok=fake, T=1.0, stats=fake, H=fake, g=fake, h=fake, grad=fake):
        return lib.umim_token_logprobs_grad(x, dtype, R, V, ld, null, tok, T, stats, H, g, h, grad, null, null)
    assert call(x=odd) == 1 and call(dtype=7) == 1 and call(ld=1004) == 1 and call(T=0.0) == 1
    assert call(V=262145, ld=262152) == 2
    assert call(g=null, h=null) == 1              # the gradient of nothing
    assert call(tok=null) == 1                    # of log probabilities of no tokens
    assert call(H=null) == 1                      # of the entropy without its value
    assert call(stats=null) == 1 and call(stats=odd) == 1
    assert call(grad=null) == 1 and call(grad=ctypes.c_void_p((1 << 20) + 8)) == 1
    assert call(R=0) == 0


def test_distill_topk_ce(lib):
    def call(ids=fake, lp=fake, R_T=3, K=8, x=fake, dtype=0, R_S=4, V=1000, ld=1000, tr=fake, sr=fake, P=4, T=1.0,
             scale=1.0, loss=fake, grad=null, ws=null, wsb=1 << 20):
        return lib.umim_distill_topk_ce(ids, lp, R_T, K, x, dtype, R_S, V, ld, tr, sr, P, null, T, 1, scale, loss, null,
                                        grad, ws, wsb, null, null)
    assert lib.umim_distill_topk_ce_workspace_size(3000, 2500) >= 3000 * 4 + 2500 * 4
    assert lib.umim_distill_topk_ce_workspace_size(0, 0) > 0
    assert lib.umim_distill_topk_ce_workspace_size(-1, 5) == 0
    assert call(K=0) == 1 and call(K=129) == 1
    assert call(R_T=-1) == 1 and call(R_S=-1) == 1 and call(P=-1) == 1
    assert call(ids=null) == 1 and call(lp=null) == 1
    assert call(x=odd) == 1 and call(dtype=3) == 1 and call(V=0) == 1 and call(ld=996) == 1
    assert call(V=300000, ld=300000) == 2
    assert call(R_S=2 ** 30 + 1) == 2 and call(P=2 ** 30 + 1) == 2
    assert call(tr=null) == 1 and call(sr=null) == 1
    assert call(T=nan) == 1 and call(scale=nan) == 1 and call(scale=math.inf) == 1
    assert call(loss=null) == 1
    assert call(grad=ctypes.c_void_p((1 << 20) + 2)) == 1
    assert call() == 5                            # no workspace
    assert call(ws=ctypes.c_void_p((1 << 20) + 16)) == 5
    assert call(ws=fake, wsb=256) == 5
