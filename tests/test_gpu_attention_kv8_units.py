"""Attention over the 8-bit cache where its rows' scales say little about what the rows are worth: scales far apart
between pages, rows of zeros (which are stored with scale 1), pages that are not there.  What a weight times its row's
scale is measured by has to come from rows that hold something, and the sum of the weights from none of that."""
import numpy as np
import pytest
import torch

import oracle
import workloads as W
from helpers import dev, umim
from kv8_helpers import PAGE, attention_bound, check_attention, i32, key_like, shared, tables, to_bf16, to_pool8

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


@pytest.mark.parametrize("kernel,B,hq", FORMS)
@pytest.mark.parametrize("size", [1.0, 0.05, 1e-12])
@pytest.mark.parametrize("share", [0, 7, 10, 13])
def test_a_sink_without_a_value(kernel, B, hq, size, share):
    """An entry with a V row of zeros and 2^share times the others' weight: the others are all of the output."""
    n = 1027
    K, V, q = plain(5, n, B, hq, size=size)
    K[3], V[3] = 0, 0
    K[3, :, 0] = np.log(2.0 ** share * n)
    Entries(6, K, V, q).check(umim(), dev(), kernel)


@pytest.mark.parametrize("kernel,B,hq", FORMS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [0, -20, -40, -60])
def test_rows_of_zeros(kernel, B, hq, D, power):
    """K and V of 2^power with rows of zeros in places: first and last of a page, a whole page, the last entry."""
    n = 333
    K, V, q = plain(7, n, B, hq, D, heads=2, size=2.0 ** power)
    K *= 2.0 ** power
    for t in (0, 15, 16, 40, n - 1):
        V[t] = 0
    V[64:80, 1] = 0
    for t in (5, 16, 70):
        K[t] = 0
    K[96:112, 0] = 0
    q *= 2.0 ** min(-power, 30)
    Entries(8, K, V, q).check(umim(), dev(), kernel, scale=2.0 ** max(0, -power - 30))


@pytest.mark.parametrize("kernel,B,hq", FORMS)
@pytest.mark.parametrize("D", [64, 128])
def test_rows_that_begin_with_zeros(kernel, B, hq, D):
    """Rows that hold something behind zeros (of both signs), beside rows that hold nothing: over pages enough for every CTA
    to have several tiles."""
    n = 128 * 160 + 77 if kernel == "tensor cores" else 777
    K, V, q = plain(21, n, B, hq, D, size=2.0 ** -30)
    K[..., :D - 3], V[..., :D - 5] = 0, -0.0
    q *= 4
    V[5::97] = 0
    K[7::89] = 0
    Entries(22, K, V, q).check(umim(), dev(), kernel)


@pytest.mark.parametrize("kernel,B,hq", FORMS[2:])
def test_zeros_beside_own_entries(kernel, B, hq):
    """A prefix whose last pages and rows hold zeros, and own entries of another size behind it."""
    n = 200
    K, V, q = plain(9, n, B, hq, size=1e-6)
    V[::3], V[160:] = 0, 0
    Entries(10, K, V, q, own=[(7 * b) % 20 for b in range(B)]).check(umim(), dev(), kernel)


@pytest.mark.parametrize("kernel,B,hq", FORMS)
@pytest.mark.parametrize("low", [0, -300])
def test_nothing_but_zeros(kernel, B, hq, low):
    """No row holds a value: zeros, however low the scores."""
    K, V, q = plain(11, 70, B, hq)
    K[..., 0] = low
    out = Entries(12, K, 0 * V, q).check(umim(), dev(), kernel)
    assert (out == 0).all()


@pytest.mark.parametrize("kernel,B,hq", FORMS)
@pytest.mark.parametrize("power", [0, -40])
def test_a_page_that_is_not_there(kernel, B, hq, power):
    """Its entries count with scores and values of zero, and set no unit for the others'."""
    K, V, q = plain(13, 100, B, hq, size=2.0 ** power)
    c = Entries(14, K, V, q)
    c.missing = [int(c.table[0, 2])]
    c.check(umim(), dev(), kernel, code=1)


@pytest.mark.parametrize("kernel,B,hq", FORMS)
def test_zeros_of_no_scale(kernel, B, hq):
    """A V row of zeros whose scale is NaN is NaN, as 0 * NaN is."""
    K, V, q = plain(15, 50, B, hq, heads=2)
    V[20] = 0
    c = Entries(16, K, V, q)
    c.scales[0, c.table[0, 1], 1, 0, 4] = 255
    got = c.run(umim(), dev(), kernel, 1.0).float().cpu().numpy()
    assert np.isnan(got[:, :hq]).all() and np.isfinite(got[:, hq:]).all()


@pytest.mark.parametrize("many", [False, True])
def test_zero_scores_are_not_moved(many):
    """A K row of zeros has a score of 0 beside keys of any size."""
    B = 40 if many else 3
    r = W.rng(17)
    n, D = 64, 64
    K, V = 2.0 ** -45 * r.standard_normal((n, 1, D)), r.standard_normal((n, 1, D))
    K[::5] = 0
    q = 2.0 ** 45 * r.standard_normal((B, 4, D)) / 4
    Entries(18, K, V, q).check(umim(), dev(), "tensor cores" if many else "pages", scale=0.25)


# the pages' kernel over 8-bit prefixes, held to what it keeps itself (not to the tensor cores' kernel's one fp16 number a
# weight): 2^-17 of a weight and 2^-40 of the largest weight times its scale
@pytest.mark.parametrize("hq,D,spread", [(4, 64, 0), (16, 128, 0), (7, 128, 10), (12, 64, 45)])
def test_pages_kernel_keeps_its_own_bound(hq, D, spread):
    r = W.rng(19 + hq)
    n, B = 777, 5
    K, V, q = plain(20 + hq, n, B, hq, D)
    V *= np.exp2(r.integers(-spread, spread + 1, V.shape[:-1]))[..., None]
    c = Entries(21, 4 * K, V, 4 * q, own=[0, 5, 16, 33, 1])
    check_attention(c.run(umim(), dev(), "pages", 0.3), *c.want("pages", 0.3))


@pytest.mark.parametrize("D,hq", [(64, 8), (128, 1), (128, 16)])
def test_rows_of_a_page_far_apart_on_the_tensor_cores(D, hq):
    """Rows of V in one page with scales up to 2^90 apart.  A row of scale f beside a largest scale of F is zeros where f is
    below 2^-31 F, 448 f <= 448 * 2^-32 F at most, and off by 2^-25 units of 2^-7 F otherwise; their mean by weights that sum
    up to 1 is off by no more than the largest of those."""
    r = W.rng(23)
    n, B = 333, 40
    K, V, q = plain(24, n, B, hq, D)
    V *= np.exp2(r.integers(-45, 46, V.shape[:-1]))[..., None]
    c = Entries(25, K, V, q)
    want, size, most, finest = c.want("tensor cores", 1.0)
    got = c.run(umim(), dev(), "tensor cores", 1.0).double().cpu().numpy()
    pages = c.table[0, :-(-n // PAGE)]
    top = 2.0 ** (int(c.scales[0, pages, 1].max()) - 127)
    assert (np.abs(got - want) <= attention_bound(want, size, most, finest, True) + 448 * 2.0 ** -32 * top).all()
