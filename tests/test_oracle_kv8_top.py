"""The largest rows of the 8-bit cache in the oracle: every finite number comes back finite, within the bound of a stored value."""
import numpy as np
import pytest

import oracle


def test_the_largest_numbers_stay_finite():
    bits = np.concatenate([np.arange(0x7f00, 0x7f80), np.arange(0xff00, 0xff80)]).astype(np.uint16)
    x = oracle.bf16.to_f64(bits)
    for b, v in zip(bits, x):   # each the largest of a row of its own
        row = np.zeros(64, np.uint16)
        row[3] = b
        c, s = oracle.kv8.quantise(row)
        got = (oracle.kv8.values(c) * oracle.kv8.scales(s))[3]
        assert abs(got) <= 240 * 2.0 ** 120 and abs(got - v) <= 2.0 ** -4 * abs(v)


@pytest.mark.parametrize("bits,code", [(0x7f6f, 0x77), (0x7f70, 0x77), (0x7f77, 0x77), (0x7f78, 0x77), (0x7f7f, 0x77),
                                       (0xff7f, 0xf7), (0x7f68, 0x76), (0x7f80, 0x7f), (0xff80, 0x7f)])
def test_codes_beside_the_largest(bits, code):
    """With e = 120: 240 = 1.875 * 2^7 (code 0x77) is the largest; 232 lies midway between 224 (0x76) and 240 and goes to the even one."""
    row = np.full(64, 0x7f7f, np.uint16)
    row[5] = bits
    c, s = oracle.kv8.quantise(row)
    assert s == 247 and c[5] == code and (c[np.arange(64) != 5] == 0x77).all()
