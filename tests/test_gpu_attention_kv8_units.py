"""Attention over the 8-bit cache where its rows' scales say little about what the rows are worth: scales far apart
between pages.  The sum of the weights has to have a measure of its own."""
import numpy as np
import pytest
import torch

import oracle
import workloads as W
from helpers import dev, umim
from kv8_helpers import PAGE, check_attention, i32, key_like, shared, tables, to_bf16, to_pool8

pytestmark = pytest.mark.gpu

NOTHING = 2.0 ** -300   # the scale that a row of zeros counts with: its weights are no unit of any other's


class Entries:
    """One list of entries (K, V as [n][heads][D] of float64) that B sequences attend to: as a cache of their own each, or
    as a prefix of all.  `wide` sends prefixes of more than 16 rows to the tensor cores' kernel."""

    def __init__(self, seed, K, V, q, own=()):
        r = W.rng(seed)
        self.n, self.heads, self.D = K.shape
        self.q = oracle.bf16.from_f32(q.astype(np.float32))
        B = len(q)
        self.own = list(own) or [0] * B
        bt, self.pages = tables(r, self.own + [self.n], spare=2)
        self.bt, self.table = bt[:B], bt[B:]
        bits = key_like(r, (1, self.pages, 2, self.heads, PAGE, self.D))
        t = np.arange(self.n)
        for which, x in enumerate((K, V)):
            bits[0, self.table[0, t // PAGE], which, :, t % PAGE] = oracle.bf16.from_f32(x.astype(np.float32))
        self.codes, self.scales = oracle.kv8.quantise(bits)
        self.missing = []

    def want(self, kernel, scale):
        """(want, size, most, finest) for check_attention, `kernel` "pages" or "tensor cores"."""
        codes, scales = self.codes.copy(), self.scales.copy()
        for p in self.missing:
            codes[:, p], scales[:, p] = 0, 127
        pool, f = oracle.kv8.pool_values(codes, scales), oracle.kv8.scales(scales)
        f = np.where((codes & 0x7f != 0).any(-1), f, NOTHING)
        table = np.array(self.table[0])
        if self.missing:
            table[table < 0] = self.missing[0]
        at, ns = [[table, t] for t in self.bt], [[self.n, n] for n in self.own]
        want, size, most, finest = oracle.kv8.attend(self.q, pool, 0, at, ns, scale, row_scales=f)
        if kernel == "tensor cores":   # in units of a page's largest scale
            F = f.copy()
            for p in range(-(-self.n // PAGE)):
                rows = f[0, table[p], 1, :, :min(PAGE, self.n - PAGE * p)]
                F[0, table[p], 1] = np.where(f[0, table[p], 1] > NOTHING, rows.max(-1)[..., None], NOTHING)
            finest = oracle.kv8.attend(self.q, pool, 0, at, ns, scale, row_scales=F)[3] + finest / 256
        return want, size, most, finest

    def run(self, m, d, kernel, scale, code=0):
        pool, status = to_pool8(m, self.codes, self.scales, d), m.new_status(d)
        q, B = to_bf16(self.q, d), len(self.q)
        prefix = np.array(self.table)
        for p in self.missing:
            prefix[prefix == p] = self.pages
        if kernel == "decode":
            assert not any(self.own)
            bt, lens = np.repeat(prefix, B, 0), [self.n] * B
            out = m.umim_decode_attention_kv8(q, pool, 0, i32(bt, d), i32(lens, d), scale=scale, dev_status=status)
        else:
            columns = 6000 if kernel == "tensor cores" else prefix.shape[1]
            full = np.full((1, columns), -1, np.int32)
            full[:, :prefix.shape[1]] = prefix
            out = m.umim_decode_attention_shared_kv8(q, pool, 0, i32(full, d), i32([self.n], d), i32(self.bt, d),
                                                     i32(self.own, d), scale=scale, dev_status=status)
        assert int(status.item()) == code
        return out

    def check(self, m, d, kernel, scale=1.0, code=0):
        out = self.run(m, d, kernel, scale, code)
        check_attention(out, *self.want("tensor cores" if kernel == "tensor cores" else "pages", scale),
                        half=kernel == "tensor cores")
        return out


# (kernel, sequences, query heads): "decode" is umim_decode_attention_kv8 with up to eight and with more query heads a KV
# head; "pages" and "tensor cores" are the shared call's kernels
FORMS = [("decode", 2, 4), ("decode", 2, 12), ("pages", 3, 4), ("tensor cores", 40, 4), ("tensor cores", 33, 1)]


def plain(seed, n, B, hq, D=64, heads=1, size=1.0):
    """(K, V, q): scores within a few units of one another, V of the given size; channel 0 of q is 1 and of K 0."""
    r = W.rng(seed)
    K, V = 0.25 * r.standard_normal((2, n, heads, D))
    q = 0.25 * r.standard_normal((B, hq * heads, D))
    K[..., 0], q[..., 0] = 0, 1
    return K, 4 * size * V, q


@pytest.mark.parametrize("kernel,B,hq", FORMS)
@pytest.mark.parametrize("gap", [60, 134, 180, 219])
@pytest.mark.parametrize("order", ["large first", "small first", "in turn"])
def test_pages_of_scales_far_apart(kernel, B, hq, gap, order):
    """Pages of V 2^gap apart and scores alike: the large ones are the output, the small ones half of the weights."""
    n = 40 * PAGE
    K, V, q = plain(1, n, B, hq)
    page = np.arange(n) // PAGE
    small = {"large first": page >= 20, "small first": page < 20, "in turn": page % 2 == 1}[order]
    V *= 2.0 ** np.where(small, min(118, gap) - gap, min(118, gap))[:, None, None]
    Entries(2, K, V, q).check(umim(), dev(), kernel)


@pytest.mark.parametrize("kernel,B,hq", FORMS)
@pytest.mark.parametrize("more", [-30, 10, 60])
def test_small_values_with_most_of_the_weight(kernel, B, hq, more):
    """The small pages' scores `more` (in log2) above the others': the weights' sum is theirs or the others', the output
    never theirs."""
    n = 40 * PAGE
    K, V, q = plain(3, n, B, hq)
    small = np.arange(n) // PAGE % 2 == 1
    V *= 2.0 ** np.where(small, -80, 80)[:, None, None]
    K[small, :, 0] = more * np.log(2)
    Entries(4, K, V, q).check(umim(), dev(), kernel)
