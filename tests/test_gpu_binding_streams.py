"""A call given a stream makes its outputs and its workspace on that stream: the zeros of a workspace made on another one
could be written while the call runs, and memory that the allocator hands on in another stream's
order could still be in use there.  (Which stream each tensor is made on is asked of the binding; no race is run.)"""
import types

import numpy as np
import pytest
import torch

import workloads as W
from helpers import case_to_dev, dev, umim
from oracle import logprobs as OL
from test_gpu_logprobs import check_forward, f64, logits

pytestmark = pytest.mark.gpu

MAKERS = ("empty", "zeros", "full", "empty_like", "zeros_like", "empty_strided")


@pytest.fixture
def made(monkeypatch):
    """The stream that is current at each call of a tensor factory."""
    streams = []
    for name in MAKERS:
        def spy(*args, _make=getattr(torch, name), **kwargs):
            streams.append(torch.cuda.current_stream().cuda_stream)
            return _make(*args, **kwargs)
        monkeypatch.setattr(torch, name, spy)
    return streams


def calls(m, dv):
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=dv)
    c = W.decode_case(5, lens=[40, 23], n_q_heads=4, n_kv_heads=2, head_dim=64, n_spans=[2, 1])
    g = case_to_dev(c, dv)
    new = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device=dv)
    mc = W.merge_case(6, vocab=50, d=512, h=1, n_spans=3)
    table, ids, offs, w = (x.to(dv) for x in (mc.table, mc.token_ids, mc.span_offsets, mc.weights))
    x = logits(7, 6, 1003, "bf16").to(dv)
    rows, tok = torch.arange(6, dtype=torch.int32, device=dv), torch.arange(6, dtype=torch.int32, device=dv)
    o = m.umim_token_logprobs(x, tok, n_top=5, vocab=1003)
    rules = torch.tensor([[1, 2, -1, -1], [3, 4, 5, -1]], dtype=torch.int32, device=dv)
    rule_table = m.umim_rules_build(rules)
    prompts = torch.tensor([[1, 2, 3, 4, 5, 9, 9, 9]], dtype=torch.int32, device=dv)
    state = m.new_suffix_state(2, dv)
    qkv = [torch.randn(9, h, 64, device=dv).bfloat16() for h in (4, 2, 2)]
    ones, cu, pair, lut = torch.ones(6, device=dv), i32(0, 4, 9), i32(1, 0), torch.ones(2, 8, device=dv)
    moved = [g[k].clone() for k in ("pool", "bt", "lens")]
    stepped, news = g["pool"].clone(), i32(1, 3)
    spans = i32(6), i32(0, 1), i32(2), i32(2)
    return dict(
        merge_spans=lambda s: m.umim_merge_spans(table, ids, offs, w, stream=s),
        kv_rollback=lambda s: m.umim_kv_rollback(*moved, g["offs"], g["st"], g["ln"], g["sk"], g["sv"], stream=s),
        decode_attention=lambda s: m.umim_decode_attention(g["q"], g["pool"], 0, g["bt"], g["lens"], stream=s),
        decode_layer_step=lambda s: m.umim_decode_layer_step(g["q"], stepped, 0, g["bt"], g["lens"], new, new, stream=s),
        prefill_attention=lambda s: m.umim_prefill_attention(*qkv, cu, stream=s),
        rules_build=lambda s: m.umim_rules_build(rules, stream=s),
        match_prompts=lambda s: m.umim_match_prompts(rule_table, prompts, merge_inputs=True, stream=s),
        match_suffix=lambda s: m.umim_match_suffix(rule_table, state, news, stream=s),
        lookup=lambda s: m.umim_lookup_surrogates(lut, pair, stream=s),
        align=lambda s: m.umim_distill_align(*spans, 10, stream=s),
        soft_ce=lambda s: m.umim_distill_soft_ce(x, x, rows, rows, vocab=1003, stream=s),
        token_logprobs=lambda s: m.umim_token_logprobs(x, tok, n_top=5, vocab=1003, stream=s),
        token_logprobs_grad=lambda s: m.umim_token_logprobs_grad(x, o["stats"], tok, ones, vocab=1003, stream=s),
        topk_ce=lambda s: m.umim_distill_topk_ce(o["top_ids"], o["top_logprobs"], x, rows, rows, vocab=1003, stream=s),
    )


def test_what_a_call_makes_is_made_on_its_stream(made):
    m, dv = umim(), dev()
    side = torch.cuda.Stream()
    here = torch.cuda.current_stream().cuda_stream
    bare = types.SimpleNamespace(cuda_stream=side.cuda_stream)   # another library's stream: its handle is enough
    for stream, handle in ((side, side.cuda_stream), (bare, side.cuda_stream), (None, here)):
        todo = calls(m, dv)        # inputs of their own for each, ready before the call
        torch.cuda.synchronize()
        for name, call in todo.items():
            del made[:]
            call(stream)
            torch.cuda.synchronize()
            assert len(made) >= 1 and set(made) == {handle}, name
            assert torch.cuda.current_stream().cuda_stream == here


def test_the_logit_calls_on_a_stream_of_their_own():
    """The same results, with all their buffers made by the calls."""
    m, dv = umim(), dev()
    V, R, K = 3001, 40, 12
    x = logits(8, R, V, "bf16")
    xd = x.to(dv)
    tokens = np.random.default_rng(1).integers(0, V, R)
    tok, rows = torch.from_numpy(tokens.astype(np.int32)).to(dv), torch.arange(R, dtype=torch.int32, device=dv)
    g = torch.ones(R, device=dv)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o = m.umim_token_logprobs(xd, tok, n_top=K, vocab=V, stream=side)
    grad = m.umim_token_logprobs_grad(xd, o["stats"], tok, g, vocab=V, stream=side)
    loss, pairs, tgrad = m.umim_distill_topk_ce(o["top_ids"], o["top_logprobs"], xd, rows, rows, vocab=V, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    check_forward(o, x, V, tokens, 1.0, K)
    again = m.umim_token_logprobs_grad(xd, o["stats"], tok, g, vocab=V)
    assert torch.equal(again[:, :V], grad[:, :V])
    want = m.umim_distill_topk_ce(o["top_ids"], o["top_logprobs"], xd, rows, rows, vocab=V)
    assert torch.equal(want[0], loss) and torch.equal(want[1], pairs) and torch.equal(want[2][:, :V], tgrad[:, :V])
    ref = OL.topk_ce(o["top_ids"].cpu().numpy(), o["top_logprobs"].cpu().numpy(), f64(x)[:, :V], np.arange(R), np.arange(R))
    assert abs(float(loss) - ref[0]) < 1e-5 * ref[0]
