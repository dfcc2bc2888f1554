"""The 8-bit cache on the GPU against the oracle: codes and scales bit by bit."""
import numpy as np
import pytest
import torch

import oracle
import workloads as W
from helpers import dev, umim
from kv8_helpers import from_pool8, i32, key_like, tables, to_bf16, to_pool8

pytestmark = pytest.mark.gpu


def rows_case(seed, lens, starts, heads, D, layers=2, fused=False, tail=0):
    """Rows of K and V for every sequence, `tail` more behind them, and a cache that holds something already."""
    r = W.rng(seed)
    d = dev()
    B, T = len(lens), int(sum(lens)) + tail
    bt, n = tables(r, [s + x for s, x in zip(starts, lens)], spare=2)
    codes = r.integers(0, 0x7f, (layers, n, 2, heads, 16, D)).astype(np.uint8)
    scales = r.integers(100, 150, (layers, n, 2, heads, 16)).astype(np.uint8)
    x = key_like(r, (T, 2, heads, D))
    dense = to_bf16(x, d)
    if fused:   # rows inside those of a projection
        wide = torch.randn((T, 3 * heads, D), device=d).bfloat16()
        wide[:, heads:] = dense.reshape(T, 2 * heads, D)
        k, v = wide[:, heads:2 * heads], wide[:, 2 * heads:]
    else:
        k, v = dense[:, 0].contiguous(), dense[:, 1].contiguous()
    return r, B, T, bt, codes, scales, x, k, v, np.concatenate([[0], np.cumsum(lens)])


def written(codes, scales, layer, bt, starts, cu, x):
    codes, scales = codes.copy(), scales.copy()
    for b in range(len(starts)):
        for t in range(cu[b], cu[b + 1]):
            e = starts[b] + t - cu[b]
            c, s = oracle.kv8.quantise(x[t])
            codes[layer, bt[b, e // 16], :, :, e % 16] = c
            scales[layer, bt[b, e // 16], :, :, e % 16] = s
    return codes, scales


CASES = [
    # lens, starts, heads, D, fused, tail
    ([1], [0], 1, 64, False, 0),
    ([1], [15], 2, 128, False, 0),
    ([33, 0, 1, 16, 0, 7], [0, 5, 16, 15, 0, 31], 8, 128, True, 0),
    ([5, 70], [100, 3], 3, 64, True, 9),
    ([0, 0, 0, 3], [1, 2, 3, 4], 5, 128, False, 2),
    ([1] * 70 + [0] * 40 + [2] * 30, [7] * 140, 1, 64, False, 0),   # more sequences than one step of the search
    ([200, 500, 333], [0, 8, 1], 8, 128, False, 0),                 # eight heads a warp
    ([513, 3], [0, 0], 7, 64, True, 0),
]


@pytest.mark.parametrize("lens,starts,heads,D,fused,tail", CASES)
def test_rows_are_written_and_read_back(lens, starts, heads, D, fused, tail):
    m, d = umim(), dev()
    r, B, T, bt, codes, scales, x, k, v, cu = rows_case(len(lens) * 7 + D, lens, starts, heads, D, fused=fused, tail=tail)
    pool = to_pool8(m, codes, scales, d)
    status = m.new_status(d)
    m.umim_kv8_write(pool, 1, i32(bt, d), i32(starts, d), k, v, cu_rows=i32(cu, d), dev_status=status)
    got = from_pool8(pool)
    want = written(codes, scales, 1, bt, starts, cu, x)
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])
    mark = [torch.full((T, heads, D), 7.0, dtype=torch.bfloat16, device=d) for _ in range(2)]
    back = m.umim_kv8_read(pool, 1, i32(bt, d), i32(starts, d), T, cu_rows=i32(cu, d), out=mark, dev_status=status)
    assert int(status.item()) == 0
    value = oracle.kv8.pool_values(*want)
    for which in range(2):
        g = back[which].double().cpu().numpy()
        for b in range(B):
            e = starts[b] + np.arange(lens[b])
            np.testing.assert_array_equal(g[cu[b]:cu[b + 1]], value[1, bt[b, e // 16], which, :, e % 16])
        assert (g[cu[-1]:] == 7).all()   # rows behind the last sequence
    a, b = m.umim_kv8_read(pool, 1, i32(bt, d), i32(starts, d), T, cu_rows=i32(cu, d))
    assert torch.equal(a[:cu[-1]], back[0][:cu[-1]]) and torch.equal(b[:cu[-1]], back[1][:cu[-1]])


@pytest.mark.parametrize("B,heads,D", [(1, 1, 64), (5, 8, 128), (70, 3, 128), (300, 8, 64)])
def test_single_rows(B, heads, D):
    m, d = umim(), dev()
    starts = [(7 * b) % 50 for b in range(B)]
    r, _, T, bt, codes, scales, x, k, v, cu = rows_case(B, [1] * B, starts, heads, D)
    pool, same = to_pool8(m, codes, scales, d), to_pool8(m, codes, scales, d)
    status = m.new_status(d)
    m.umim_kv8_write(pool, 0, i32(bt, d), i32(starts, d), k, v, dev_status=status)
    want = written(codes, scales, 0, bt, starts, cu, x)
    np.testing.assert_array_equal(from_pool8(pool)[0], want[0])
    np.testing.assert_array_equal(from_pool8(pool)[1], want[1])
    m.umim_kv8_write(same, 0, i32(bt, d), i32(starts, d), k, v, cu_rows=i32(cu, d), dev_status=status)
    assert torch.equal(same.values.view(torch.uint8), pool.values.view(torch.uint8))
    a, b = m.umim_kv8_read(pool, 0, i32(bt, d), i32(starts, d), B, dev_status=status)
    c, e = m.umim_kv8_read(pool, 0, i32(bt, d), i32(starts, d), B, cu_rows=i32(cu, d), dev_status=status)
    assert torch.equal(a, c) and torch.equal(b, e) and int(status.item()) == 0


@pytest.mark.parametrize("D", [64, 128])
def test_every_bf16_number(D):
    """Rows over all exponents, NaN and infinities, zeros of both signs and the ends of the range."""
    m, d = umim(), dev()
    r = W.rng(5)
    n = 65536 // D
    x = np.arange(65536).astype(np.uint16).reshape(n, 1, D)             # neighbours: finite and infinite rows
    y = np.where(r.random((n, 1, D)) < 0.1, x.reshape(-1)[r.permutation(65536)].reshape(n, 1, D), x & 0x0fff | 0x3000)
    y[0], y[1], y[2, 0, 3:] = 0, 0x8000, 0
    y[3], y[4], y[5, 0, 1:] = 0x7f7f, 0x0001, 0x7fc0
    y = y.astype(np.uint16)
    bt, pages = tables(r, [n])
    pool = m.Kv8Pool.zeros(1, pages, 1, D, d)
    status = m.new_status(d)
    m.umim_kv8_write(pool, 0, i32(bt, d), i32([0], d), to_bf16(x, d), to_bf16(y, d), cu_rows=i32([0, n], d),
                     dev_status=status)
    codes, scales = from_pool8(pool)
    e = np.arange(n)
    for which, rows in enumerate((x, y)):
        c, s = oracle.kv8.quantise(rows)
        np.testing.assert_array_equal(codes[0, bt[0, e // 16], which, :, e % 16], c)
        np.testing.assert_array_equal(scales[0, bt[0, e // 16], which, :, e % 16], s)
    assert int(status.item()) == 0


def test_read_of_any_code_and_scale():
    m, d = umim(), dev()
    D = 64
    codes = np.arange(256, dtype=np.uint8).reshape(1, 1, 1, 1, 4, 64).repeat(64, 1).repeat(2, 2).repeat(4, 4)
    scales = np.arange(256, dtype=np.uint8)[np.arange(64 * 2 * 16) // 4 % 256].reshape(1, 64, 2, 1, 16)
    pool = to_pool8(m, codes, scales, d)
    k, v = m.umim_kv8_read(pool, 0, i32(np.arange(64)[None], d), i32([0], d), 1024, cu_rows=i32([0, 1024], d))
    want = oracle.kv8.pool_values(codes, scales)[0, :, :, 0].transpose(1, 0, 2, 3).reshape(2, 1024, 1, D)
    for got, w in zip((k, v), want):
        with np.errstate(over="ignore"):
            f = torch.from_numpy(w).float().bfloat16().double().numpy()   # exact but at the ends of the range
        np.testing.assert_array_equal(got.double().cpu().numpy(), f)


def test_bad_rows_are_left_out_and_reported():
    m, d = umim(), dev()
    lens, starts = [3, 2, 4, 5, 2], [14, 0, 30, 0, 0]
    r, B, T, bt, codes, scales, x, k, v, cu = rows_case(9, lens, starts, 2, 64, layers=1)
    bt = bt[:, :2].copy()            # sequence 2's entries 32, 33 have no page
    bt[0, 1] = codes.shape[1]        # a page that is not there: entry 16 of sequence 0
    bt[3, 0] = -1                    # nor here: all of sequence 3
    starts[4] = -1                   # no entry at all
    want = (codes.copy(), scales.copy())
    places = [(0, 0, 14, bt[0, 0]), (1, 0, 15, bt[0, 0]), (3, 1, 0, bt[1, 0]), (4, 1, 1, bt[1, 0]), (5, 2, 14, bt[2, 1]),
              (6, 2, 15, bt[2, 1])]
    for t, b, slot, page in places:
        want[0][0, page, :, :, slot], want[1][0, page, :, :, slot] = oracle.kv8.quantise(x[t])
    pool = to_pool8(m, codes, scales, d)
    status = m.new_status(d)
    m.umim_kv8_write(pool, 0, i32(bt, d), i32(starts, d), k, v, cu_rows=i32(cu, d), dev_status=status)
    assert int(status.item()) == 1
    np.testing.assert_array_equal(from_pool8(pool)[0], want[0])
    np.testing.assert_array_equal(from_pool8(pool)[1], want[1])
    mark = [torch.full((T, 2, 64), 7.0, dtype=torch.bfloat16, device=d) for _ in range(2)]
    status.zero_()
    m.umim_kv8_read(pool, 0, i32(bt, d), i32(starts, d), T, cu_rows=i32(cu, d), out=mark, dev_status=status)
    assert int(status.item()) == 1
    good = [t for t, *_ in places]
    for g in mark:
        assert (g[[t for t in range(T) if t not in good]] == 7).all() and not (g[good] == 7).all()


@pytest.mark.parametrize("cu", [[0, 5, 3, 9], [1, 2, 3, 9], [0, 3, 5, 12]])
def test_bad_offsets_are_reported(cu):
    m, d = umim(), dev()
    r, B, T, bt, codes, scales, x, k, v, _ = rows_case(10, [9, 9, 9], [0, 0, 0], 1, 64, layers=1)
    pool = to_pool8(m, codes, scales, d)
    status = m.new_status(d)
    m.umim_kv8_write(pool, 0, i32(bt, d), i32([0, 0, 0], d), k[:9], v[:9], cu_rows=i32(cu, d), dev_status=status)
    assert int(status.item()) == 1
    got = from_pool8(pool)[0]
    used = [bt[b, 0] for b in range(3)]
    others = [p for p in range(codes.shape[1]) if p not in used]
    np.testing.assert_array_equal(got[:, others], codes[:, others])


def test_rows_past_2_31_values():
    """A cache of more than 2^31 values, rows at its end."""
    m, d = umim(), dev()
    heads, D, n = 8, 128, 70000                      # 2^31 / 32768 = 65536
    pool = m.Kv8Pool.zeros(1, n, heads, D, d)
    bt = i32([[n - 1, 65535, 65536, 3]], d)
    r = W.rng(11)
    x = key_like(r, (2, 64, heads, D))
    status = m.new_status(d)
    m.umim_kv8_write(pool, 0, bt, i32([0], d), to_bf16(x[0], d), to_bf16(x[1], d), cu_rows=i32([0, 64], d),
                     dev_status=status)
    k, v = m.umim_kv8_read(pool, 0, bt, i32([0], d), 64, cu_rows=i32([0, 64], d), dev_status=status)
    assert int(status.item()) == 0
    for got, rows in zip((k, v), x):
        c, s = oracle.kv8.quantise(rows)
        np.testing.assert_array_equal(got.double().cpu().numpy(), oracle.kv8.values(c) * oracle.kv8.scales(s)[..., None])
    assert int(pool.values.view(torch.uint8).count_nonzero(dim=(0, 2, 3, 4, 5)).count_nonzero()) == 4


APPEND = [
    # seed, lens, layers, heads, D, merging
    (1, [0], 1, 1, 64, False),
    (2, [0, 1, 15, 16, 17, 31, 32, 33], 4, 2, 64, True),
    (3, list(range(0, 64, 3)), 32, 8, 128, True),       # eight CTAs a sequence
    (4, [5, 16, 47, 63], 33, 8, 128, True),             # more rows than they hold at once
    (5, list(range(1, 200)), 1, 4, 128, True),
]


@pytest.mark.parametrize("seed,lens,layers,heads,D,merging", APPEND)
def test_append_merge_steps(seed, lens, layers, heads, D, merging):
    """Steps of a decode loop on the 8-bit cache, some sequences merging: all that it holds after every step."""
    m, d = umim(), dev()
    r = W.rng(20 + seed)
    B, steps = len(lens), 4
    bt, n = tables(r, lens, columns=-(-(max(lens) + steps) // 16) + 1, spare=B * (steps + 1))
    used = set(bt[bt >= 0].tolist())
    free = [p for p in range(n) if p not in used]
    codes = r.integers(0, 0x7f, (layers, n, 2, heads, 16, D)).astype(np.uint8)
    scales = r.integers(100, 150, codes.shape[:-1]).astype(np.uint8)
    pool = to_pool8(m, codes, scales, d)
    g_bt, g_lens, o_lens = i32(bt, d), i32(lens, d), np.array(lens)
    status = m.new_status(d)
    for step in range(steps):
        new_pages = np.array([free.pop() for _ in range(B)], np.int32)
        nk, nv = key_like(r, (2, B, layers, heads, D))
        merge_k = np.where(r.random(B) < 0.4, r.integers(1, 17, B), 0) if merging else np.zeros(B, int)
        merge_k = np.minimum(merge_k, o_lens + 1)
        k = int((merge_k > 0).sum())
        rows = r.permutation(max(1, k))[np.maximum(np.cumsum(merge_k > 0) - 1, 0)]
        sk, sv = key_like(r, (2, max(1, k), layers, heads, D))
        kw = dict(merge_k=i32(merge_k, d), merge_row=i32(rows, d), surrogate_k=to_bf16(sk, d),
                  surrogate_v=to_bf16(sv, d)) if merging else {}
        rel = m.umim_kv8_append_merge(pool, g_bt, g_lens, to_bf16(nk, d), to_bf16(nv, d), i32(new_pages, d),
                                      dev_status=status, **kw)
        codes, scales, bt, o_lens, released, rejected = oracle.kv8.append_merge(
            codes, scales, bt, o_lens, nk, nv, new_pages, merge_k, rows, sk, sv)
        assert rejected == [] and int(status.item()) == 0
        np.testing.assert_array_equal(g_bt.cpu().numpy(), bt)
        np.testing.assert_array_equal(g_lens.cpu().numpy(), o_lens)
        np.testing.assert_array_equal(rel.cpu().numpy(), released)
        got = from_pool8(pool)
        np.testing.assert_array_equal(got[0], codes)
        np.testing.assert_array_equal(got[1], scales)


def test_append_merge_leaves_bad_sequences_alone():
    m, d = umim(), dev()
    r = W.rng(30)
    lens = np.array([64, -1, 5, 5, 16, 20, 3, 7, 16], np.int32)
    bt, n = tables(r, [64, 5, 5, 5, 16, 20, 3, 7, 16], columns=4, spare=4)
    bt[5, 0] = n                                     # the page that a merge reaches back to
    merge_k = np.array([0, 0, 7, 2, 0, 6, -1, 17, 0], np.int32)
    rows = np.array([0, 0, 0, 9, 0, 0, 0, 0, 0], np.int32)
    new_pages = np.array([0, 0, 0, 0, n, 0, 0, 0, n - 1], np.int32)
    codes, scales = np.zeros((2, n, 2, 2, 16, 64), np.uint8), np.full((2, n, 2, 2, 16), 127, np.uint8)
    nk, nv, sk, sv = key_like(r, (4, 9, 2, 2, 64))
    want = oracle.kv8.append_merge(codes, scales, bt, lens, nk, nv, new_pages, merge_k, rows, sk, sv)
    assert want[5] == list(range(8))
    pool, status = to_pool8(m, codes, scales, d), m.new_status(d)
    g_bt, g_lens = i32(bt, d), i32(lens, d)
    m.umim_kv8_append_merge(pool, g_bt, g_lens, to_bf16(nk, d), to_bf16(nv, d), i32(new_pages, d), i32(merge_k, d),
                            i32(rows, d), to_bf16(sk, d), to_bf16(sv, d), dev_status=status)
    assert int(status.item()) == 1
    np.testing.assert_array_equal(from_pool8(pool)[0], want[0])
    np.testing.assert_array_equal(g_bt.cpu().numpy(), want[2])
    np.testing.assert_array_equal(g_lens.cpu().numpy(), want[3])


def test_binding_refuses():
    m, d = umim(), dev()
    pool = m.Kv8Pool.zeros(1, 4, 2, 64, d)
    bt, start = i32([[0, 1]], d), i32([0], d)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=d)
    cu = i32([0, 3], d)
    write = lambda k, v, cu=cu, bt=bt, start=start: m.umim_kv8_write(pool, 0, bt, start, k, v, cu_rows=cu)
    write(k, k)
    for bad in (k.float(), k[:, :1], k[..., :32], k.cpu(), k[:1].expand(3, 2, 64), k.transpose(0, 1).contiguous().transpose(0, 1)):
        with pytest.raises(ValueError):
            write(bad, bad)
    with pytest.raises(ValueError):
        write(k, torch.zeros((3, 4, 64), dtype=torch.bfloat16, device=d)[:, :2])   # another stride
    with pytest.raises(ValueError):
        write(k, k, cu=i32([0, 3, 3], d))
    with pytest.raises(ValueError):
        write(k, k, cu=cu.long())
    with pytest.raises(ValueError):
        write(k, k, bt=bt[0])
    with pytest.raises(m.UmimError) as e:
        m.umim_kv8_write(pool, 1, bt, start, k, k, cu_rows=cu)
    assert e.value.code == 1
