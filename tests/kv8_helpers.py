"""Cases of the 8-bit cache and of attention over shared prefixes."""
import numpy as np
import torch

import oracle
import workloads as W

PAGE = 16


def tables(r, lens, columns=None, spare=0):
    """(block table [n][columns] of pages in any order, -1 behind a sequence's last; pages of the pool)."""
    need = [-(-int(n) // PAGE) for n in lens]
    columns = max([1, columns or 0] + need)
    total = max(1, sum(need) + spare)
    order = iter(r.permutation(total)[:sum(need)])
    bt = np.full((len(lens), columns), -1, np.int32)
    for b, n in enumerate(need):
        bt[b, :n] = [next(order) for _ in range(n)]
    return bt, total


def key_like(r, shape, std=1.0):
    """bf16 bits: normal numbers, every eleventh channel six times as large, rows of many sizes."""
    x = r.standard_normal(shape) * std * np.exp2(r.integers(-3, 4, shape[:-1]))[..., None]
    x[..., 3::11] *= 6
    return oracle.bf16.from_f32(x.astype(np.float32))


def pool_bits(r, layers, pages, heads, D):
    return key_like(r, (layers, pages, 2, heads, PAGE, D))


def to_bf16(bits, d):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).to(d)


def to_pool8(m, codes, scales, d):
    return m.Kv8Pool(torch.from_numpy(np.ascontiguousarray(codes)).to(d).view(torch.float8_e4m3fn),
                     torch.from_numpy(np.ascontiguousarray(scales)).to(d).view(torch.float8_e8m0fnu))


def from_pool8(pool):
    return pool.values.view(torch.uint8).cpu().numpy(), pool.scales.view(torch.uint8).cpu().numpy()


def i32(x, d):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype=np.int32))).to(d)


def attention_bound(want, size, most, finest, half):
    """How far an output may be from its value in 64 bits.

    The output is rounded once, 2^-8 of itself.  A score is an fp32 sum of at most 128 products in the tensor core,
    whose additions are off by at most 2^-22 of the sum of |q||K| each in a chain of 16 (one for every 8 products
    or fewer): 2^-18 of it, and its scaling and the subtraction of the maximum take 2^-22 of |score| <= that sum.  A
    weight is off by that much of itself, and by 2^-20 for exp2f and its fp32 factors, and its two parts (bf16, the
    coarser) hold it to 2^-17; the row sum is off by as much again.  Weighted by |V| that is
        2 * (2^-17 + 2^-17 + 2^-17 * most) * size,
    doubled for partial results merged with weights of their own.

    Over the 8-bit cache a weight times its row's scale is an fp16 number and an fp16 remainder in units of 2^-15 of
    the largest of them (or of a piece's largest, which is smaller): the remainder is a multiple of 2^-24 of such a
    unit, so however small the weight, 2^-25 * 2^-15 = 2^-40 of the largest one may be missing, of every row's
    |V| / scale.  That is 2^-40 * finest; it shows where the rows of the large weights hold zeros in a column.

    half: over a prefix of many rows in the 8-bit cache a weight is one fp16 number, off by 2^-12 of itself (the row
    sum is made of the weights before that).  Operands there are in units of their page's largest scale F, so it is
    weight * F whose largest is (after the running maximum) 2^7 or more units and that is a multiple of 2^-24 of one:
    2^-25 * 2^-7 = 2^-32 of the largest weight * F may be missing of every row's |V| / F, a row's own scale of which
    is F at most.  SharedCase's `finest` is that sum, and 2^-8 of the rows' (2^-32 * 2^-8 = 2^-40).  (Rows are exact there while
    their scales lie within 2^22 of their page's largest: test_values_far_apart_on_the_tensor_cores has others.)"""
    eps = 4 * (2.0 ** -16 + 2.0 ** -17 * most[..., None]) + (2.0 ** -12 if half else 0)
    return 2.0 ** -8 * np.abs(want) + eps * size + 2.0 ** (-32 if half else -40) * finest + 1e-30


def check_attention(got, want, size, most, finest, half=False):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    err = np.abs(got - want)
    bound = attention_bound(want, size, most, finest, half)
    bad = ok & (err > bound)
    assert not bad.any(), (np.argwhere(bad)[:5], err[bad][:5], bound[bad][:5])


class SharedCase:
    """Groups of sequences over prefixes, in a 16- and an 8-bit cache of the same values."""

    def __init__(self, seed, prefix_lens, groups, lens, Hq, Hkv, D, layers=1, offsets=None, wide=False):
        r = W.rng(seed)
        self.prefix_lens, self.lens, self.Hkv = list(prefix_lens), list(lens), Hkv
        B = len(lens)
        self.offsets = np.concatenate([[0], np.cumsum(groups)]) if offsets is None else np.asarray(offsets)
        bt, self.pages = tables(r, list(lens) + list(prefix_lens), spare=3)
        self.bt, self.prefix_bt = bt[:B], bt[B:]
        if wide:   # a table wide enough that prefixes of many rows go to the tensor cores' kernel, however short
            full = np.full((len(prefix_lens), 6000), -1, np.int32)
            full[:, :self.prefix_bt.shape[1]] = self.prefix_bt
            self.prefix_bt = full
        self.bits = pool_bits(r, layers, self.pages, Hkv, D)
        self.codes, self.scales = oracle.kv8.quantise(self.bits)
        self.q = key_like(r, (B, Hq, D))
        for b in range(0, B, 3):   # rows of other sizes
            self.q[b] = oracle.bf16.from_f32(oracle.bf16.to_f64(self.q[b]).astype(np.float32) * 0.125)

    def want(self, bits, layer=0, scale=None):
        pool = oracle.bf16.to_f64(self.bits) if bits == 16 else oracle.kv8.pool_values(self.codes, self.scales)
        at, ns = [], []
        for b in range(len(self.lens)):
            at.append([self.bt[b]])
            ns.append([self.lens[b]])
            for i in range(len(self.prefix_lens)):
                if self.offsets[i] <= b < self.offsets[i + 1]:
                    at[b].insert(0, self.prefix_bt[i])
                    ns[b].insert(0, self.prefix_lens[i])
        if bits == 16:
            return oracle.kv8.attend(self.q, pool, layer, at, ns, scale)
        own = oracle.kv8.scales(self.scales)
        most_of = own.copy()   # V's scales: the largest of a prefix's page, over the entries that it has
        for table, n in zip(self.prefix_bt, self.prefix_lens):
            for p in range(-(-n // PAGE)):
                most_of[:, table[p], 1] = own[:, table[p], 1, :, :min(PAGE, n - PAGE * p)].max(-1)[..., None]
        want, size, most, finest = oracle.kv8.attend(self.q, pool, layer, at, ns, scale, row_scales=own)
        return want, size, most, oracle.kv8.attend(self.q, pool, layer, at, ns, scale, row_scales=most_of)[3] + finest / 256

    def args(self, m, bits, d):
        pool = to_bf16(self.bits, d) if bits == 16 else to_pool8(m, self.codes, self.scales, d)
        return dict(q=to_bf16(self.q, d), pool=pool, prefix_table=i32(self.prefix_bt, d),
                    prefix_lens=i32(self.prefix_lens, d), block_table=i32(self.bt, d), seq_lens=i32(self.lens, d),
                    prefix_offsets=i32(self.offsets, d))


def shared(m, bits):
    return m.umim_decode_attention_shared if bits == 16 else m.umim_decode_attention_shared_kv8
