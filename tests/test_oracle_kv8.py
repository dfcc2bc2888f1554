"""What pins the oracle of the 8-bit cache: the library's e4m3 cast, closed forms,
the 16-bit cache's append and rollback, and decode attention over joined tables."""
import numpy as np
import pytest
import torch

import oracle
import workloads as W
from helpers import oracle_append_merge
from kv8_helpers import SharedCase, key_like, pool_bits, tables


def f32_bits(x):
    return oracle.bf16.from_f32(np.asarray(x, dtype=np.float32))


def test_table_is_the_librarys_e4m3():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(oracle.kv8.values(codes), want)
    assert np.nanmax(oracle.kv8.E4M3) == 448


def test_rounding_is_the_librarys():
    """Every bf16 number up to 448, ties among them."""
    bits = np.arange(0x43e1, dtype=np.uint16)          # 0x43e0 is 448
    x = oracle.bf16.to_f64(bits)
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(oracle.kv8._codes(x), want)
    np.testing.assert_array_equal(oracle.kv8._codes(-x), want | 0x80)


@pytest.mark.parametrize("most,e", [(448, 0), (450, 1), (449.9, 1), (224, -1), (225, 0), (1.0, -8), (1.75, -8),
                                    (1.7578125, -7), (2.0 ** -126, -100), (2.0 ** -133, -100),
                                    (3.3895313892515355e38, 120), (2.0 ** -92, -100), (2.0 ** -91, -99)])
def test_scale_is_the_smallest_that_holds_the_row(most, e):
    row = np.zeros(64)
    row[5], row[7] = -most, most / 2
    codes, scale = oracle.kv8.quantise(f32_bits(row))
    assert int(scale) == e + 127
    most = oracle.bf16.to_f64(f32_bits(most))
    assert most <= 448 * 2.0 ** e and (e == -100 or most > 448 * 2.0 ** (e - 1))
    if e > -100:
        assert abs(oracle.kv8.values(codes)[5]) > 224 * (1 - 2.0 ** -4)


def test_rows_without_numbers():
    row = np.zeros(128)
    c, s = oracle.kv8.quantise(f32_bits(row))
    assert s == 127 and (c == 0).all()
    c, s = oracle.kv8.quantise(f32_bits(-row))
    assert s == 127 and (c == 0x80).all()              # the sign of zero stays
    row[:] = np.nan
    row[3], row[4] = np.inf, -np.inf
    c, s = oracle.kv8.quantise(f32_bits(row))
    assert s == 127 and (c == 0x7f).all()
    row[9] = 3.0                                        # and one: the row's scale is that number's
    c, s = oracle.kv8.quantise(f32_bits(row))
    assert s == 127 - 7 and (c[np.arange(128) != 9] == 0x7f).all() and oracle.kv8.values(c)[9] == 384


def test_error_bounds():
    x = key_like(W.rng(1), (300, 128))
    c, s = oracle.kv8.quantise(x)
    v, got = oracle.bf16.to_f64(x), oracle.kv8.values(c) * oracle.kv8.scales(s)[:, None]
    assert (np.abs(got - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10 * oracle.kv8.scales(s)[:, None])).all()
    c2, s2 = oracle.kv8.quantise(f32_bits(got))          # what is stored once is stored again, scale included
    keep = s2 == s                                       # (or half of it, where the largest was rounded down to 224)
    np.testing.assert_array_equal(c2[keep], c[keep])
    np.testing.assert_array_equal(oracle.kv8.values(c2) * oracle.kv8.scales(s2)[:, None], got)


def test_append_merge_is_the_16_bit_caches():
    """Written rows apart, an update of the 8-bit cache is the append and rollback of the 16-bit one."""
    r = W.rng(2)
    lens = np.array([1, 15, 16, 17, 31, 32, 33, 48, 0], np.int32)
    B, layers, H, D = len(lens), 2, 2, 64
    bt, n = tables(r, lens, columns=4, spare=B)
    free = [p for p in range(n) if p not in set(bt.ravel().tolist())]
    new_pages = np.array(free[:B], np.int32)
    merge_k = np.array([2, 0, 1, 3, 4, 2, 0, 16, 0], np.int32)
    rows = np.cumsum(merge_k > 0) - 1
    bits = pool_bits(r, layers, n, H, D)
    nk, nv = key_like(r, (2, B, layers, H, D))
    sk, sv = key_like(r, (2, int((merge_k > 0).sum()), layers, H, D))
    codes, scales = oracle.kv8.quantise(bits)
    got = oracle.kv8.append_merge(codes, scales, bt, lens, nk, nv, new_pages, merge_k, rows, sk, sv)
    want = oracle_append_merge(bits, bt, lens, nk, nv, new_pages, merge_k, sk, sv)
    assert got[5] == []
    np.testing.assert_array_equal(got[2], want[1])
    np.testing.assert_array_equal(got[3], want[2])
    np.testing.assert_array_equal(got[4], want[3])
    for b in range(B):
        t = np.arange(int(want[2][b]))
        at = (slice(None), want[1][b, t // 16], slice(None), slice(None), t % 16)
        c, s = oracle.kv8.quantise(want[0][at])
        np.testing.assert_array_equal(got[0][at], c)
        np.testing.assert_array_equal(got[1][at], s)


def test_append_merge_rejects():
    r = W.rng(3)
    lens = np.array([64, -1, 5, 5, 16], np.int32)
    bt, n = tables(r, [64, 5, 5, 5, 16], columns=4, spare=4)
    bits = pool_bits(r, 1, n, 1, 64)
    x = key_like(r, (5, 1, 1, 64))
    codes, scales = oracle.kv8.quantise(bits)
    out = oracle.kv8.append_merge(codes, scales, bt, lens, x, x, [0, 0, 0, 0, n], [0, 0, 7, 2, 0], [0, 0, 0, 9, 0], x, x)
    assert out[5] == [0, 1, 2, 3, 4]
    np.testing.assert_array_equal(out[0], codes)
    np.testing.assert_array_equal(out[2], bt)


def test_shared_attention_is_attention_over_joined_tables():
    c = SharedCase(4, prefix_lens=[48, 0, 32], groups=[2, 1, 2], lens=[5, 0, 17, 1, 33], Hq=4, Hkv=2, D=64)
    out, size, most, finest = c.want(16)
    joined = np.full((5, 6), -1, np.int32)
    lens = []
    for b, i in enumerate([0, 0, 1, 2, 2]):
        n = c.prefix_lens[i] // 16
        joined[b, :n] = c.prefix_bt[i, :n]
        joined[b, n:n + 3] = c.bt[b][:3]
        lens.append(c.prefix_lens[i] + c.lens[b])
    np.testing.assert_allclose(out, oracle.decode_attention(c.q, c.bits, 0, joined, lens), rtol=1e-12, atol=1e-14)
    assert (size >= np.abs(out) - 1e-12).all() and (most > 0).all() and (finest == 0).all()


def test_attention_over_nothing_is_zero():
    c = SharedCase(5, prefix_lens=[0], groups=[2], lens=[0, 3], Hq=2, Hkv=1, D=64)
    out, *_ = c.want(8)
    assert (out[0] == 0).all() and (out[1] != 0).any()
