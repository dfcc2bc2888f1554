"""Groups of uneven sizes on the tensor cores' kernel, which runs where a batch's groups have rows enough on average: large and small
ones together, prefixes and groups that are empty, sequences of no prefix, one query head a KV head."""
import pytest

import workloads as W
from helpers import dev, umim
from kv8_helpers import SharedCase, check_attention, shared

pytestmark = pytest.mark.gpu

CASES = [
    # prefix lens, sequences up to each prefix's first and last, own lens, Hq, Hkv, D
    ([300, 40, 0, 77, 500], [0, 90, 91, 94, 94, 130], 130, 8, 2, 64),       # 90, 1, 3 behind nothing, none, 36
    ([129, 1000], [7, 70, 110], 125, 16, 2, 128),                          # 7 and 15 of no prefix
    ([640, 64], [0, 100, 180], 180, 4, 4, 128),                            # one query head a KV head
    ([257, 0, 16, 15], [3, 60, 100, 160, 161], 170, 5, 1, 64),             # the last group of five rows
    ([2049], [60, 120], 140, 7, 1, 128),
    ([31, 33], [0, 33, 66], 66, 32, 2, 64),                                # eight sequences a tile of rows
]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("prefix_lens,offsets,B,hq,hkv,d", CASES)
def test_uneven_groups(prefix_lens, offsets, B, hq, hkv, d, bits):
    m, dv = umim(), dev()
    r = W.rng(B + hq)
    c = SharedCase(B, prefix_lens, None, r.integers(0, 40, B).tolist(), hq, hkv, d, layers=2, offsets=offsets, wide=True)
    status = m.new_status(dv)
    m.trace_start()
    got = shared(m, bits)(layer=1, dev_status=status, **c.args(m, bits, dv))
    m.trace_stop()
    assert "attention.prefix" in [label for label, _ in m.trace_read()]
    check_attention(got, *c.want(bits, 1), half=bits == 8)
    assert int(status.item()) == 0
