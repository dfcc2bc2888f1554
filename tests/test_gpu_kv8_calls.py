"""Calls of the 8-bit cache and of shared prefixes as programs make them: rows at odd places, in graphs, on side
streams, on caller's buffers, on the debug build."""
import os

import numpy as np
import pytest
import torch

import oracle
import workloads as W
from helpers import dev, umim
from kv8_helpers import SharedCase, check_attention, from_pool8, i32, key_like, shared, tables, to_bf16, to_pool8

pytestmark = pytest.mark.gpu


def wide_rows(rows, before, behind, d):
    """rows [T][H][D] of bits inside rows that hold `before` and `behind` more values."""
    T, H, D = rows.shape
    x = torch.full((T, before + H * D + behind), 3.0, dtype=torch.bfloat16, device=d)
    x[:, before:before + H * D] = to_bf16(rows, d).view(T, H * D)
    return x, x[:, before:before + H * D].view(T, H, D)


@pytest.mark.parametrize("before,behind", [(0, 0), (8, 0), (0, 8), (8, 8), (24, 32)])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_16_bytes_apart(before, behind, D):
    """Rows that start on 16- but not on 32-byte boundaries."""
    m, d = umim(), dev()
    r = W.rng(before + D)
    T, H = 37, 3
    bt, n = tables(r, [T])
    x = key_like(r, (2, T, H, D))
    (_, k), (_, v) = wide_rows(x[0], before, behind, d), wide_rows(x[1], before, behind, d)
    pool, status = m.Kv8Pool.zeros(1, n, H, D, d), m.new_status(d)
    cu, start = i32([0, T], d), i32([0], d)
    m.umim_kv8_write(pool, 0, i32(bt, d), start, k, v, cu_rows=cu, dev_status=status)
    e = np.arange(T)
    codes, scales = from_pool8(pool)
    for which in range(2):
        c, s = oracle.kv8.quantise(x[which])
        np.testing.assert_array_equal(codes[0, bt[0, e // 16], which, :, e % 16], c)
        np.testing.assert_array_equal(scales[0, bt[0, e // 16], which, :, e % 16], s)
    (fk, ok), (fv, ov) = wide_rows(0 * x[0], before, behind, d), wide_rows(0 * x[1], before, behind, d)
    m.umim_kv8_read(pool, 0, i32(bt, d), start, T, cu_rows=cu, out=(ok, ov), dev_status=status)
    a, b = m.umim_kv8_read(pool, 0, i32(bt, d), start, T, cu_rows=cu)
    assert torch.equal(ok, a) and torch.equal(ov, b) and int(status.item()) == 0
    for full in (fk, fv):   # what lies between the rows stays
        assert (full[:, :before] == 3).all() and (full[:, before + H * D:] == 3).all()


def test_a_step_in_a_graph():
    """Tokens written, appended, read and attended to in one captured step, replayed on other values."""
    m, d = umim(), dev()
    r = W.rng(80)
    B, H, D, layers = 5, 2, 64, 2
    lens = np.array([3, 15, 31, 40, 0], np.int32)
    bt, n = tables(r, lens, columns=4, spare=2 * B)
    free = [p for p in range(n) if p not in set(bt.ravel().tolist())]
    new_pages = np.array(free[:B], np.int32)
    codes, scales = oracle.kv8.quantise(key_like(r, (layers, n, 2, H, 16, D)))
    pool, first = to_pool8(m, codes, scales, d), to_pool8(m, codes, scales, d)
    g_bt, g_lens = i32(bt, d), i32(lens, d)
    nk, nv = torch.zeros((2, B, layers, H, D), dtype=torch.bfloat16, device=d)
    q, merge_k = torch.zeros((B, 4, D), dtype=torch.bfloat16, device=d), i32([0] * B, d)
    rows = i32(range(B), d)
    ws = m.workspace(m.umim_decode_attention_kv8_workspace_size(B, 4, H, D), d)
    out, pages = torch.empty_like(q), i32(new_pages, d)

    def step():
        m.umim_kv8_append_merge(pool, g_bt, g_lens, nk, nv, pages, merge_k, rows, nv, nk)
        m.umim_decode_attention_kv8(q, pool, 1, g_bt, g_lens, out=out, workspace_buf=ws)

    def reset():
        for a, b in ((pool.values, first.values), (pool.scales, first.scales)):
            a.view(torch.uint8).copy_(b.view(torch.uint8))
        g_bt.copy_(i32(bt, d)), g_lens.copy_(i32(lens, d))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        reset()
        x = key_like(r, (2, B, layers, H, D))
        qb = key_like(r, (B, 4, D))
        k = np.minimum(np.where(r.random(B) < 0.5, 3, 0), lens + 1)
        nk.copy_(to_bf16(x[0], d)), nv.copy_(to_bf16(x[1], d)), q.copy_(to_bf16(qb, d)), merge_k.copy_(i32(k, d))
        graph.replay()
        c, s, obt, ol, _, _ = oracle.kv8.append_merge(codes, scales, bt, lens, x[0], x[1], new_pages, k, np.arange(B),
                                                      x[1], x[0])
        np.testing.assert_array_equal(from_pool8(pool)[0], c)
        np.testing.assert_array_equal(g_lens.cpu().numpy(), ol)
        check_attention(out, *oracle.kv8.attend(qb, oracle.kv8.pool_values(c, s), 1, [[t] for t in obt], [[y] for y in ol],
                                                row_scales=oracle.kv8.scales(s)))


def test_side_stream_makes_what_the_call_needs():
    m, d = umim(), dev()
    c = SharedCase(81, [40], [3], [5, 0, 9], 8, 2, 128)
    side = torch.cuda.Stream(d)
    for bits in (16, 8):
        a = c.args(m, bits, d)
        torch.cuda.synchronize()
        out = shared(m, bits)(layer=0, stream=side, **a)
        side.synchronize()
        check_attention(out, *c.want(bits), half=bits == 8)
    pool = to_pool8(m, c.codes, c.scales, d)
    bt, start = i32(c.bt, d), i32([0, 0, 0], d)
    torch.cuda.synchronize()
    k, v = m.umim_kv8_read(pool, 0, bt[:1], start[:1], 3, cu_rows=i32([0, 3], d), stream=side)
    side.synchronize()
    want = oracle.kv8.pool_values(c.codes, c.scales)[0, c.bt[0, 0]]
    np.testing.assert_array_equal(k.double().cpu().numpy(), want[0].transpose(1, 0, 2)[:3])
    np.testing.assert_array_equal(v.double().cpu().numpy(), want[1].transpose(1, 0, 2)[:3])


@pytest.mark.parametrize("bits", [16, 8])
def test_callers_buffers(bits):
    m, d = umim(), dev()
    c = SharedCase(82, [70], [40], [b % 7 for b in range(40)], 8, 2, 64, wide=True)
    a = c.args(m, bits, d)
    size = m.umim_decode_attention_shared_workspace_size(40, 1, 8, 2, 64)
    ws = torch.full((size + 512,), 0xff, dtype=torch.uint8, device=d)   # nothing in it has to be zero
    out = torch.empty_like(a["q"])
    assert shared(m, bits)(layer=0, out=out, workspace_buf=ws[:size], **a) is out
    check_attention(out, *c.want(bits), half=bits == 8)
    assert (ws[size:] == 0xff).all()
    for bad in (ws[:size - 256], ws[16:]):
        with pytest.raises(m.UmimError) as e:
            shared(m, bits)(layer=0, workspace_buf=bad, **a)
        assert e.value.code == 5
    with pytest.raises(ValueError):
        shared(m, bits)(layer=0, out=out[:, :4], **a)
    with pytest.raises(m.UmimError) as e:   # rows of q that no copy can start on
        q = torch.zeros(a["q"].numel() + 8, dtype=torch.bfloat16, device=d)[4:-4].view(a["q"].shape)
        shared(m, bits)(layer=0, **{**a, "q": q})
    assert e.value.code == 1


@pytest.mark.parametrize("bits", [16, 8])
def test_two_streams_at_once_on_the_tensor_cores(bits):
    m, d = umim(), dev()
    cases = [SharedCase(83 + i, [900 + i], [50], [b % 9 for b in range(50)], 8, 2, 128, wide=True) for i in range(2)]
    args = [c.args(m, bits, d) for c in cases]
    want = [shared(m, bits)(layer=0, **a) for a in args]
    streams = [torch.cuda.Stream(d) for _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [shared(m, bits)(layer=0, stream=s, **a) for a, s in zip(args, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))


def test_empty_batches():
    m, d = umim(), dev()
    pool = m.Kv8Pool.zeros(1, 2, 1, 64, d)
    none = torch.zeros((0, 1, 64), dtype=torch.bfloat16, device=d)
    bt0, i0 = torch.zeros((0, 1), dtype=torch.int32, device=d), i32([], d)
    m.umim_kv8_write(pool, 0, bt0, i0, none, none)
    k, v = m.umim_kv8_read(pool, 0, i32([[0]], d), i32([0], d), 0, cu_rows=i32([0, 0], d))
    assert k.shape == (0, 1, 64)
    q = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device=d)
    assert m.umim_decode_attention_kv8(q, pool, 0, bt0, i0).shape == q.shape
    assert m.umim_decode_attention_shared_kv8(q, pool, 0, i32([[0]], d), i32([3], d), bt0, i0).shape == q.shape
    rel = m.umim_kv8_append_merge(pool, bt0, i0, none.view(0, 1, 1, 64), none.view(0, 1, 1, 64))
    assert rel.numel() == 0


@pytest.fixture
def debug_library():
    import paper_2609_27233_gb300 as umim_pkg
    from paper_2609_27233_gb300 import _lib, build
    if not os.path.exists(_lib.DEBUG_LIB_PATH):
        build.build(variants=("debug",))
    umim_pkg.use_debug_library(True)
    try:
        yield
    finally:
        umim_pkg.use_debug_library(False)


def test_debug_build(debug_library):
    """The same comparisons on the build that checks its own indexes; no site reports."""
    import test_gpu_attention_kv8 as A
    import test_gpu_kv8 as R
    assert umim().umim_debug_build() == 1
    for case in R.CASES[:5]:
        R.test_rows_are_written_and_read_back(*case)
    R.test_bad_rows_are_left_out_and_reported()
    for case in R.APPEND[:4]:
        R.test_append_merge_steps(*case)
    for case in A.CASES[:9]:
        A.test_attention(*case)
    for bits in (16, 8):
        for case in A.SHARED:
            for wide in (False, True):
                A.test_shared(*case, bits, wide)
        for many in (False, True):
            A.test_bad_arguments_on_the_device(bits, many)
