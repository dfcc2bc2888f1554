"""Rows at the top of bf16's range in the 8-bit cache: written by either call, every finite number reads back finite."""
import numpy as np
import pytest
import torch

import oracle
import workloads as W
from helpers import dev, umim
from kv8_helpers import from_pool8, i32, tables, to_bf16

pytestmark = pytest.mark.gpu


def rows_at_the_top(D):
    """Rows whose largest is each of the 128 largest magnitudes, some beside NaN and infinities."""
    r = W.rng(D)
    x = r.integers(0x7e00, 0x7f00, (256, 1, D)).astype(np.uint16)
    x[:128, 0, 5], x[128:, 0, D - 1] = np.arange(0x7f00, 0x7f80), np.arange(0xff00, 0xff80)
    x[3::7, 0, 9], x[4::7, 0, 10] = 0x7f80, 0x7fc0
    return x


@pytest.mark.parametrize("D", [64, 128])
def test_the_largest_numbers_read_back_finite(D):
    m, d = umim(), dev()
    x = rows_at_the_top(D)
    bt, pages = tables(W.rng(1), [256])
    pool, status = m.Kv8Pool.zeros(1, pages, 1, D, d), m.new_status(d)
    cu, start = i32([0, 256], d), i32([0], d)
    m.umim_kv8_write(pool, 0, i32(bt, d), start, to_bf16(x, d), to_bf16(x[::-1].copy(), d), cu_rows=cu, dev_status=status)
    codes, scales = from_pool8(pool)
    e = np.arange(256)
    for which, rows in enumerate((x, x[::-1])):
        c, s = oracle.kv8.quantise(rows)
        np.testing.assert_array_equal(codes[0, bt[0, e // 16], which, :, e % 16], c)
        np.testing.assert_array_equal(scales[0, bt[0, e // 16], which, :, e % 16], s)
    k, v = m.umim_kv8_read(pool, 0, i32(bt, d), start, 256, cu_rows=cu, dev_status=status)
    assert int(status.item()) == 0
    for got, rows in ((k, x), (v, x[::-1])):
        g, want = got.double().cpu().numpy(), oracle.bf16.to_f64(rows)
        finite = np.isfinite(want)
        np.testing.assert_array_equal(np.isfinite(g), finite)
        assert (np.abs(g - want)[finite] <= 2.0 ** -4 * np.abs(want)[finite]).all()


def test_appended_rows_too():
    m, d = umim(), dev()
    D, B = 64, 256
    x = rows_at_the_top(D).reshape(B, 1, 1, D)
    pool = m.Kv8Pool.zeros(1, B, 1, D, d)
    bt, lens = torch.full((B, 1), -1, dtype=torch.int32, device=d), i32([0] * B, d)
    m.umim_kv8_append_merge(pool, bt, lens, to_bf16(x, d), to_bf16(x, d), i32(range(B), d))
    codes, scales = from_pool8(pool)
    c, s = oracle.kv8.quantise(x[:, 0])
    for which in range(2):
        np.testing.assert_array_equal(codes[0, :, which, :, 0], c)
        np.testing.assert_array_equal(scales[0, :, which, :, 0], s)
