"""Decode attention over the 8-bit cache and over shared prefixes (both caches) on
the GPU against the oracle, within a bound derived from the roundings."""
import numpy as np
import pytest
import torch

import oracle
import workloads as W
from helpers import dev, umim
from kv8_helpers import SharedCase, attention_bound, check_attention, i32, key_like, shared, tables, to_bf16, to_pool8

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, seed, lens, Hq, Hkv, D, layers=1, sizes=0):
        r = W.rng(seed)
        self.lens = list(lens)
        self.bt, self.pages = tables(r, lens, spare=2)
        bits = key_like(r, (layers, self.pages, 2, Hkv, 16, D))
        if sizes:   # rows whose scales are far apart
            f = oracle.bf16.to_f64(bits) * np.exp2(r.integers(-sizes, sizes + 1, bits.shape[:-1]))[..., None]
            f[:, :, 0] = oracle.bf16.to_f64(bits)[:, :, 0]
            bits = oracle.bf16.from_f32(f.astype(np.float32))
        self.codes, self.scales = oracle.kv8.quantise(bits)
        self.q = key_like(r, (len(lens), Hq, D))
        self.q[::2] = oracle.bf16.from_f32(oracle.bf16.to_f64(self.q[::2]).astype(np.float32) * 0.125)

    def want(self, layer=0, scale=None):
        return oracle.kv8.attend(self.q, oracle.kv8.pool_values(self.codes, self.scales), layer,
                                 [[t] for t in self.bt], [[n] for n in self.lens], scale,
                                 row_scales=oracle.kv8.scales(self.scales))

    def run(self, m, d, layer=0, code=0, **kw):
        status = m.new_status(d)
        out = m.umim_decode_attention_kv8(to_bf16(self.q, d), to_pool8(m, self.codes, self.scales, d), layer,
                                          i32(self.bt, d), i32(self.lens, d), dev_status=status, **kw)
        assert int(status.item()) == code
        return out


CASES = [
    ([1], 1, 1, 64), ([1], 16, 1, 128), ([16, 17, 15, 0, 1, 2, 31, 33], 8, 2, 128), ([0, 0, 40, 0], 8, 8, 64),
    ([432], 8, 2, 64), ([700, 1200, 64], 16, 16, 128), ([300, 2500], 16, 1, 64), ([300, 999], 32, 2, 128),
    ([3000, 3], 28, 4, 128), ([1001, 16 * 60], 8, 4, 64), ([5, 900], 10, 2, 128), ([77, 300], 36, 4, 64),
    (list(range(130)), 4, 1, 64),
]


@pytest.mark.parametrize("lens,hq,hkv,d", CASES)
def test_attention(lens, hq, hkv, d):
    c = Case(sum(lens) + hq, lens, hq, hkv, d, layers=2)
    for layer in (0, 1):
        check_attention(c.run(umim(), dev(), layer), *c.want(layer))


@pytest.mark.parametrize("hq,hkv,d,sizes", [(8, 2, 128, 10), (16, 1, 64, 10), (4, 1, 128, 45), (12, 1, 128, 45)])
def test_rows_of_values_of_other_sizes(hq, hkv, d, sizes):
    """V rows of scales 2^-sizes .. 2^sizes: a weight and its value's scale may lie far apart."""
    c = Case(91, [200, 33, 700], hq, hkv, d, sizes=sizes)
    check_attention(c.run(umim(), dev()), *c.want())


@pytest.mark.parametrize("hq", [4, 12])
def test_explicit_scale_and_sharp_softmax(hq):
    c = Case(92, [500, 77], hq, 1, 128)
    for scale in (0.25, 3.0, 1e-3):
        check_attention(c.run(umim(), dev(), scale=scale), *c.want(scale=scale))


def test_queries_of_all_sizes():
    c = Case(93, [60] * 12, 4, 2, 64)
    f = oracle.bf16.to_f64(c.q) * np.exp2(np.array([-140, -100, -86, -60, -20, -10, 0, 3, 5, -126, -90, 1]))[:, None, None]
    c.q = oracle.bf16.from_f32(f.astype(np.float32))
    c.q[3] = 0
    c.q[4, :, ::2] = 0x0001                       # the smallest of all
    check_attention(c.run(umim(), dev()), *c.want())
    c.codes[:, :, 0], c.scales[:, :, 0] = 0x30, 127 + 100   # and keys to match the smallest
    got = c.run(umim(), dev(), scale=1e-2)
    assert torch.isfinite(got.float()[[0, 1, 2, 9, 10]]).all()


@pytest.mark.parametrize("hq", [4, 12])
def test_garbage_past_the_end_is_ignored(hq):
    c = Case(94, [21, 5, 16, 1], hq, 1, 128)
    for b, n in enumerate(c.lens):
        for t in range(n, -(-n // 16) * 16):
            c.codes[:, c.bt[b, t // 16], :, :, t % 16] = 0x7f if b % 2 else 0xff
            c.scales[:, c.bt[b, t // 16], :, :, t % 16] = 255
    check_attention(c.run(umim(), dev()), *c.want())


@pytest.mark.parametrize("hq", [4, 12])
@pytest.mark.parametrize("which", ["key", "value", "key scale", "value scale"])
def test_nan_stays_with_its_sequence(hq, which):
    c = Case(95, [40, 40], hq, 2, 64)
    kv = 0 if "key" in which else 1
    if "scale" in which:
        c.scales[0, c.bt[0, 1], kv, 0, 3] = 255
    else:
        c.codes[0, c.bt[0, 1], kv, 0, 3, 7] = 0x7f
    want = c.want()
    got = c.run(umim(), dev()).float().cpu().numpy()
    half = hq // 2
    assert np.isnan(got[0, :half] if which != "value" else got[0, :half, 7]).all()
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want[0]))
    check_attention(torch.from_numpy(got[1:]), *(x[1:] for x in want))


def test_a_bad_page_reads_as_zeros_and_a_bad_length_as_none():
    m, d = umim(), dev()
    c = Case(96, [40, 20, 30], 8, 2, 128)
    bt = c.bt.copy()
    c.bt[0, 1], c.bt[1, 0] = c.pages, -1
    out = c.run(m, d, code=1)
    c.codes[0, bt[0, 1]], c.codes[0, bt[1, 0]] = 0, 0
    c.bt = bt
    check_attention(out, *c.want())
    c.lens[1] = 16 * c.bt.shape[1] + 1
    got = c.run(m, d, code=1).float()
    assert (got[1] == 0).all() and (got[0] != 0).any()
    c.lens[1] = -5
    assert (c.run(m, d, code=1).float()[1] == 0).all()


def test_more_sequences_than_a_block_plans():
    c = Case(97, [(7 * b) % 23 for b in range(4200)], 2, 1, 64)
    check_attention(c.run(umim(), dev()), *c.want())


def test_dequantised_cache_and_16_bit_attention_agree():
    """umim_kv8_read's rows in a 16-bit cache: the same attention but for rounding."""
    m, d = umim(), dev()
    c = Case(98, [1500, 700, 31], 32, 8, 128)
    pool = oracle.bf16.from_f32(oracle.kv8.pool_values(c.codes, c.scales).astype(np.float32))
    a = m.umim_decode_attention(to_bf16(c.q, d), to_bf16(pool, d), 0, i32(c.bt, d), i32(c.lens, d))
    b = c.run(m, d)
    check_attention(a, *c.want())
    check_attention(b, *c.want())


def test_cache_past_2_31_values():
    m, d = umim(), dev()
    r = W.rng(99)
    heads, D, n = 8, 128, 70000
    pool = m.Kv8Pool.zeros(1, n, heads, D, d)
    pages = [n - 1, 65535, 65536, 5, 69000]
    codes, scales = oracle.kv8.quantise(key_like(r, (1, 5, 2, heads, 16, D)))
    pool.values.view(torch.uint8)[:, pages] = torch.from_numpy(codes).to(d)
    pool.scales.view(torch.uint8)[:, pages] = torch.from_numpy(scales).to(d)
    q = key_like(r, (1, 32, D))
    got = m.umim_decode_attention_kv8(to_bf16(q, d), pool, 0, i32([pages], d), i32([75], d))
    check_attention(got, *oracle.kv8.attend(q, oracle.kv8.pool_values(codes, scales), 0, [[np.arange(5)]], [[75]],
                                            row_scales=oracle.kv8.scales(scales)))


# ---------------------------------------------------------------------------
# shared prefixes
# ---------------------------------------------------------------------------
SHARED = [
    # prefix lens, groups, own lens, Hq, Hkv, D
    ([1], [1], [0], 1, 1, 64),
    ([0], [2], [0, 5], 4, 2, 128),
    ([100], [2], [0, 33], 8, 2, 64),
    ([33], [5], [1, 16, 17, 0, 40], 28, 4, 128),
    ([15, 16, 17], [1, 1, 1], [3, 0, 16], 2, 1, 64),
    ([300, 0, 77, 5], [3, 2, 0, 4], [5, 1, 0, 100, 0, 7, 30, 16, 2], 16, 2, 128),
    ([1000], [9], [4] * 9, 16, 1, 128),                          # rows that fill blocks unevenly
    ([640, 64], [7, 30], [(5 * b) % 40 for b in range(37)], 8, 8, 64),
    ([2000], [70], [(3 * b) % 20 for b in range(70)], 8, 2, 128),
    ([129, 511], [33, 40], [(3 * b) % 20 for b in range(73)], 16, 4, 64),
    ([257], [130], [b % 3 for b in range(130)], 5, 1, 128),
]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("prefix_lens,groups,lens,hq,hkv,d", SHARED)
def test_shared(prefix_lens, groups, lens, hq, hkv, d, bits, wide):
    m, dv = umim(), dev()
    c = SharedCase(len(lens) + hq, prefix_lens, groups, lens, hq, hkv, d, layers=2, wide=wide)
    status = m.new_status(dv)
    for layer in (0, 1):
        check_attention(shared(m, bits)(layer=layer, dev_status=status, **c.args(m, bits, dv)), *c.want(bits, layer), half=bits == 8)
    if len(groups) == 1:
        a = c.args(m, bits, dv)
        del a["prefix_offsets"]
        check_attention(shared(m, bits)(layer=1, dev_status=status, scale=0.3, **a), *c.want(bits, 1, 0.3), half=bits == 8)
    assert int(status.item()) == 0


@pytest.mark.parametrize("bits", [16, 8])
def test_sequences_of_no_prefix(bits):
    m, dv = umim(), dev()
    c = SharedCase(40, [50, 20], None, [5, 0, 30, 7, 0, 12], 8, 2, 64, offsets=[1, 3, 4])
    check_attention(shared(m, bits)(layer=0, **c.args(m, bits, dv)), *c.want(bits), half=bits == 8)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("many", [False, True])
def test_garbage_past_the_ends(bits, many):
    m, dv = umim(), dev()
    B = 64 if many else 3
    c = SharedCase(41, [37], [B], [(7 * b) % 19 for b in range(B)], 16, 2, 128, wide=many)
    for table, n in [(c.prefix_bt[0], 37)] + list(zip(c.bt, c.lens)):
        for t in range(n, -(-n // 16) * 16):
            c.bits[:, table[t // 16], :, :, t % 16] = 0x7fc0 if t % 2 else 0xff80
            c.codes[:, table[t // 16], :, :, t % 16] = 0x7f
            c.scales[:, table[t // 16], :, :, t % 16] = 255
    check_attention(shared(m, bits)(layer=0, **c.args(m, bits, dv)), *c.want(bits), half=bits == 8)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("many", [False, True])
def test_bad_arguments_on_the_device(bits, many):
    """Lengths, offsets and pages that are not there: reported, and what the header says instead."""
    m, dv = umim(), dev()
    B = 64 if many else 6
    c = SharedCase(42, [50, 40], [B - 2, 2], [5] * B, 8, 2, 64, wide=many)

    def run(**change):
        a = c.args(m, bits, dv)
        a.update({k: i32(v, dv) for k, v in change.items()})
        status = m.new_status(dv)
        out = shared(m, bits)(layer=0, dev_status=status, **a)
        assert int(status.item()) == 1
        return out
    cols = c.prefix_bt.shape[1]
    full = c.want(bits)
    for bad in (-1, 16 * cols + 1):
        got = run(prefix_lens=[bad, 40])
        c.prefix_lens[0] = 0
        check_attention(got, *c.want(bits), half=bits == 8)
        c.prefix_lens[0] = 50
    got = run(prefix_offsets=[0, B - 2, B + 1])          # the second prefix has nobody
    keep = c.offsets
    c.offsets = np.array([0, B - 2, B - 2])
    check_attention(got, *c.want(bits), half=bits == 8)
    c.offsets = keep
    got = run(prefix_offsets=[B - 2, 3, B])              # (B - 2, B - 2, B)
    c.offsets = np.array([B - 2, B - 2, B])
    check_attention(got, *c.want(bits), half=bits == 8)
    c.offsets = keep
    bt = c.prefix_bt.copy()
    bt[0, 1] = c.pages
    got = run(prefix_table=bt)
    z = c.prefix_bt[0, 1]
    c.bits[:, z], c.codes[:, z] = 0, 0
    check_attention(got, *c.want(bits), half=bits == 8)
    assert not np.array_equal(full[0], c.want(bits)[0])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("many", [False, True])
def test_nan_in_a_prefix(bits, many):
    m, dv = umim(), dev()
    B = 66 if many else 4
    c = SharedCase(43, [50, 40], [B - 2, 2], [5] * B, 8, 2, 64, wide=many)
    c.bits[0, c.prefix_bt[0, 1], 0, 1, 2, 5], c.codes[0, c.prefix_bt[0, 1], 0, 1, 2, 5] = 0x7fc0, 0x7f
    got = shared(m, bits)(layer=0, **c.args(m, bits, dv)).float().cpu().numpy()
    assert np.isnan(got[:B - 2, 4:]).all() and np.isfinite(got[:, :4]).all() and np.isfinite(got[B - 2:]).all()
    check_attention(torch.from_numpy(got[:, :4].copy()), *(x[:, :4] for x in c.want(bits)), half=bits == 8)


@pytest.mark.parametrize("d", [64, 128])
def test_values_far_apart_on_the_tensor_cores(d):
    """Rows of V in one page with scales up to 2^30 apart.  The operands are multiples of 2^-24 in units of 2^-7 of the
    page's largest scale: a value is off by 2^-32 of that at most, and so is their mean by weights that sum up to 1."""
    m, dv = umim(), dev()
    c = SharedCase(45, [333], [40], [(5 * b) % 20 for b in range(40)], 8, 2, d, wide=True)
    f = oracle.bf16.to_f64(c.bits)
    f[:, :, 1] *= np.exp2(W.rng(46).integers(-11, 12, f[:, :, 1].shape[:-1]))[..., None]
    c.codes, c.scales = oracle.kv8.quantise(oracle.bf16.from_f32(f.astype(np.float32)))
    s = c.scales[:, :, 1].astype(int)
    assert (s.max(-1) - s.min(-1)).max() <= 31
    want, size, most, finest = c.want(8)
    got = shared(m, 8)(layer=0, **c.args(m, 8, dv))
    err = np.abs(got.double().cpu().numpy() - want)
    top = 2.0 ** (s.max() - 127)
    assert (err <= attention_bound(want, size, most, finest, True) + 2.0 ** -32 * top).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("B", [3, 70])
def test_no_entries_at_all(bits, B):
    """Tables without columns, or lengths of zero: zeros, and nothing is reported; a prefix alone needs no own table."""
    m, dv = umim(), dev()
    c = SharedCase(47, [90], [B], [0] * B, 8, 2, 128, wide=B > 3)
    a, status = c.args(m, bits, dv), m.new_status(dv)
    none = torch.zeros((B, 0), dtype=torch.int32, device=dv)
    check_attention(shared(m, bits)(layer=0, dev_status=status, **{**a, "block_table": none}), *c.want(bits), half=bits == 8)
    zero = i32([0], dv)
    for change in ({}, {"block_table": none}, {"prefix_table": none[:1]}, {"block_table": none, "prefix_table": none[:1]}):
        out = torch.ones_like(a["q"])
        shared(m, bits)(layer=0, dev_status=status, out=out, **{**a, "prefix_lens": zero, **change})
        assert (out == 0).all()
    assert int(status.item()) == 0


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("wide", [False, True])
def test_many_prefixes(bits, wide):
    m, dv = umim(), dev()
    n = 40 if wide else 200
    r = W.rng(44)
    groups = r.integers(0, 40 if wide else 4, n)
    B = int(groups.sum())
    c = SharedCase(44, r.integers(0, 200 if wide else 60, n).tolist(), groups, r.integers(0, 20, B).tolist(), 4, 2, 64,
                   wide=wide)
    check_attention(shared(m, bits)(layer=0, **c.args(m, bits, dv)), *c.want(bits), half=bits == 8)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("B", [3, 70])
def test_graphs_share_a_workspace(bits, B):
    """Two captured calls on one workspace, replayed in turn, with an eager call between: each its own answer."""
    m, dv = umim(), dev()
    cases = [SharedCase(50 + i, [200 + 90 * i], [B], [(3 + i) * b % 20 for b in range(B)], 8, 2, 128, wide=B > 3)
             for i in range(2)]
    ws = m.workspace(m.umim_decode_attention_shared_workspace_size(B, 1, 8, 2, 128), dv)
    args = [c.args(m, bits, dv) for c in cases]
    outs = [torch.empty_like(a["q"]) for a in args]
    eager = [shared(m, bits)(layer=0, workspace_buf=ws, **a).clone() for a in args]
    graphs = []
    for a, o in zip(args, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            shared(m, bits)(layer=0, workspace_buf=ws, out=o, **a)
        graphs.append(g)
    for _ in range(3):
        for i in (0, 1, 1, 0):
            outs[i].zero_()
            graphs[i].replay()
            shared(m, bits)(layer=0, workspace_buf=ws, **args[1 - i])
            assert torch.equal(outs[i], eager[i])
    check_attention(outs[0], *cases[0].want(bits), half=bits == 8)


def test_calls_at_once_on_two_streams():
    m, dv = umim(), dev()
    c = [Case(60, [900, 40], 8, 2, 128), Case(61, [33, 1200], 8, 2, 128)]
    want = [x.run(m, dv) for x in c]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(dv) for _ in c]
    args = [(to_bf16(x.q, dv), to_pool8(m, x.codes, x.scales, dv), 0, i32(x.bt, dv), i32(x.lens, dv)) for x in c]
    torch.cuda.synchronize()
    for _ in range(20):
        got = [m.umim_decode_attention_kv8(*a, stream=s) for a, s in zip(args, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("B", [3, 70])
def test_results_do_not_change_between_calls(bits, B):
    m, dv = umim(), dev()
    c = SharedCase(62, [3000], [B], [b % 30 for b in range(B)], 16, 2, 128, wide=B > 3)
    a = c.args(m, bits, dv)
    first = shared(m, bits)(layer=0, **a)
    for _ in range(10):
        assert torch.equal(shared(m, bits)(layer=0, **a), first)


def test_binding_refuses():
    m, dv = umim(), dev()
    c = SharedCase(63, [20], [2], [3, 4], 4, 2, 64)
    for bits in (16, 8):
        a = c.args(m, bits, dv)
        for name, bad in (("q", a["q"].float()), ("q", a["q"][:, :, :32]), ("q", a["q"].transpose(0, 1)),
                          ("prefix_lens", a["prefix_lens"].long()), ("seq_lens", a["seq_lens"][:1]),
                          ("prefix_offsets", a["prefix_offsets"][:1]), ("block_table", a["block_table"][:1]),
                          ("prefix_table", a["prefix_table"][0]), ("block_table", a["block_table"].cpu())):
            with pytest.raises(ValueError):
                shared(m, bits)(layer=0, **{**a, name: bad})
        with pytest.raises(m.UmimError) as e:
            shared(m, bits)(layer=1, **a)
        assert e.value.code == 1


# ---------------------------------------------------------------------------
# a decode loop on the 8-bit cache
# ---------------------------------------------------------------------------
def test_loop_prompts_steps_and_merges():
    """Prompts written, steps appended with merges, and after each step attention of every sequence: over its own
    cache, and, the same prompt shared, over prefix and continuation."""
    m, dv = umim(), dev()
    r = W.rng(70)
    B, layers, Hq, Hkv, D, P, steps = 5, 2, 8, 2, 128, 37, 6
    prompt = key_like(r, (2, layers, P, Hkv, D))
    bt, n = tables(r, [0] * B + [P], columns=4, spare=B * (steps + 2))
    own, pre = bt[:B], bt[B:]
    free = [p for p in range(n) if p not in set(bt.ravel().tolist())]
    codes, scales = np.zeros((layers, n, 2, Hkv, 16, D), np.uint8), np.full((layers, n, 2, Hkv, 16), 127, np.uint8)
    pool, status = to_pool8(m, codes, scales, dv), m.new_status(dv)
    for layer in range(layers):
        m.umim_kv8_write(pool, layer, i32(pre, dv), i32([0], dv), to_bf16(prompt[0, layer], dv),
                         to_bf16(prompt[1, layer], dv), cu_rows=i32([0, P], dv), dev_status=status)
        for t in range(P):
            c, s = oracle.kv8.quantise(prompt[:, layer, t])
            codes[layer, pre[0, t // 16], :, :, t % 16], scales[layer, pre[0, t // 16], :, :, t % 16] = c, s
    lens = np.zeros(B, np.int32)
    g_bt, g_lens = i32(own, dv), i32(lens, dv)
    for step in range(steps):
        nk, nv, sk, sv = key_like(r, (4, B, layers, Hkv, D))
        new_pages = np.array([free.pop() for _ in range(B)], np.int32)
        merge_k = np.minimum(np.where(r.random(B) < 0.4, 2, 0), lens + 1)
        rows = np.arange(B)
        m.umim_kv8_append_merge(pool, g_bt, g_lens, to_bf16(nk, dv), to_bf16(nv, dv), i32(new_pages, dv),
                                i32(merge_k, dv), i32(rows, dv), to_bf16(sk, dv), to_bf16(sv, dv), dev_status=status)
        codes, scales, own, lens, _, _ = oracle.kv8.append_merge(codes, scales, own, lens, nk, nv, new_pages, merge_k,
                                                                 rows, sk, sv)
        values, powers = oracle.kv8.pool_values(codes, scales), oracle.kv8.scales(scales)
        q = key_like(r, (B, Hq, D))
        for layer in range(layers):
            got = m.umim_decode_attention_kv8(to_bf16(q, dv), pool, layer, g_bt, g_lens, dev_status=status)
            check_attention(got, *oracle.kv8.attend(q, values, layer, [[t] for t in own], [[x] for x in lens],
                                                    row_scales=powers))
            got = m.umim_decode_attention_shared_kv8(to_bf16(q, dv), pool, layer, i32(pre, dv), i32([P], dv), g_bt,
                                                     g_lens, dev_status=status)
            check_attention(got, *oracle.kv8.attend(q, values, layer, [[pre[0], t] for t in own], [[P, x] for x in lens],
                                                    row_scales=powers))
    assert int(status.item()) == 0
