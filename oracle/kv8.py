"""The 8-bit paged cache of the oracle (test infrastructure only): rows quantised
to e4m3 with a power of two a row, the cache update of a decode step on such a
cache, and attention over shared prefixes.

The paper keeps its cache in 16 bits; the format is this library's.  A row x of D
values is stored as c_i = e4m3(x_i / 2^e), rounded to nearest, ties to even, with
the smallest whole e such that max |x_i| <= 448 * 2^e over the finite x_i, kept in
[-100, 120], and e = 0 for a row without any but zeros.  NaN and infinities are
stored as NaN, finite magnitudes above 240 * 2^120 as that (256 * 2^120 is no
bf16 number).  The e8m0 code of 2^e is e + 127.

e4m3: sign, four exponent bits (bias 7), three fraction bits; no infinities, all
ones is NaN, so the largest number is 1.75 * 2^8 = 448 and the smallest 2^-9.
Codes are turned into numbers by a table, and numbers into codes by the nearest
entry of that table.
"""
import numpy as np

from . import attention, bf16


def _table():
    v = np.zeros(128)
    for c in range(127):
        e, m = c >> 3, c & 7
        v[c] = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
    v[127] = np.nan
    return v


E4M3 = _table()
_MID = (E4M3[:126] + E4M3[1:127]) / 2


def values(codes):
    """e4m3 codes (uint8) as float64."""
    c = np.asarray(codes, dtype=np.uint8)
    return np.where(c & 0x80, -1.0, 1.0) * E4M3[c & 0x7f]


def scales(codes):
    """e8m0 codes (uint8) as float64: 2^(code - 127), NaN for 255."""
    c = np.asarray(codes, dtype=np.uint8).astype(np.int64)
    return np.where(c == 255, np.nan, np.ldexp(1.0, c - 127))


def _codes(y):
    """The nearest e4m3 code of |y| <= 448, ties to the even code."""
    a = np.abs(y)
    lo = np.searchsorted(_MID, a, side="left")          # a on a midpoint: the code below it
    tie = (lo < 126) & (a == _MID[np.minimum(lo, 125)])
    return (np.where(tie & (lo % 2 == 1), lo + 1, lo) | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def quantise(bits):
    """(codes uint8 [..][D], scale codes uint8 [..]) of rows of bf16 bits [..][D]."""
    x = bf16.to_f64(bits)
    finite = np.isfinite(x)
    most = np.where(finite, np.abs(x), 0).max(-1)
    e = np.zeros(most.shape, dtype=np.int64)
    for i in np.ndindex(*most.shape):
        if most[i] > 0:
            k = -100
            while k < 120 and most[i] > 448 * 2.0 ** k:
                k += 1
            e[i] = k
    with np.errstate(invalid="ignore"):
        y = np.clip(np.where(finite, x, 0), -240 * 2.0 ** 120, 240 * 2.0 ** 120) / np.ldexp(1.0, e)[..., None]
    return np.where(finite, _codes(y), 0x7f).astype(np.uint8), (e + 127).astype(np.uint8)


def pool_values(codes, scale_codes):
    """A cache [layers][pages][2][Hkv][P][D] as float64."""
    return values(codes) * scales(scale_codes)[..., None]


def attend(q_bits, pool, layer, tables, lens, scale=None, page_size=16, row_scales=None):
    """Attention of q [B][Hq][D] over a cache in float64 [layers][pages][2][Hkv][P][D].  tables[b] and lens[b] are
    lists of page lists and lengths: b attends to all of their entries.  Returns (out [B][Hq][D], the sum of the
    weights times |V|, of the same shape, the largest sum |q||K| times the scale [B][Hq], and, with row_scales
    [layers][pages][2][Hkv][P], the largest weight times its V row's scale times the sum of |V| / scale, [B][Hq][D],
    else zeros)."""
    q = bf16.to_f64(q_bits)
    B, Hq, D = q.shape
    Hkv = pool.shape[3]
    G = Hq // Hkv
    scale = scale if scale else 1.0 / np.sqrt(D)
    out, size, most, finest = np.zeros((B, Hq, D)), np.zeros((B, Hq, D)), np.zeros((B, Hq)), np.zeros((B, Hq, D))
    for b in range(B):
        rows, powers = [], []
        for pages, n in zip(tables[b], lens[b]):
            t = np.arange(n)
            at = (layer, np.asarray(pages)[t // page_size], slice(None), slice(None), t % page_size)
            rows.append(pool[at])   # [n][2][Hkv][D]
            if row_scales is not None:
                powers.append(row_scales[at][:, 1])
        rows = np.concatenate(rows)
        if len(rows) == 0:
            continue
        for h in range(Hq):
            K, V = rows[:, 0, h // G], rows[:, 1, h // G]
            out[b, h], w = attention.attend(q[b, h], K, V, scale)
            size[b, h] = w @ np.abs(V)
            most[b, h] = scale * (np.abs(K) @ np.abs(q[b, h])).max()
            if row_scales is not None:
                f = np.concatenate(powers)[:, h // G]
                finest[b, h] = (w * f).max() * (np.abs(V) / f[:, None]).sum(0)
    return out, size, most, finest


def append_merge(codes, scale_codes, block_table, seq_lens, new_k, new_v, new_pages, merge_k, merge_row, sur_k, sur_v,
                 page_size=16):
    """One decode step on an 8-bit cache: for sequence b with L entries and k = merge_k[b], the new entry at slot L
    (k = 0) or surrogate row merge_row[b] at slot L + 1 - k in place of the last k entries, the new one among them.
    Rows are bf16 bits [B or rows][layers][Hkv][D].  Returns (codes, scale_codes, table, lens, released, rejected)."""
    codes, scale_codes = codes.copy(), scale_codes.copy()
    bt, lens = np.array(block_table), np.array(seq_lens)
    n_pages = codes.shape[1]
    released, rejected = np.full(len(lens), -1, np.int32), []
    for b in range(len(lens)):
        L, k = int(lens[b]), int(merge_k[b])
        row = bt[b].copy()
        if L < 0 or L >= bt.shape[1] * page_size or k < 0 or k > min(16, L + 1):
            rejected.append(b)
            continue
        if L % page_size == 0:
            row[L // page_size] = new_pages[b]
        slot = L + 1 - k if k else L
        opened, page = row[L // page_size], row[slot // page_size]
        if not (0 <= opened < n_pages and 0 <= page < n_pages) or (k and not 0 <= merge_row[b] < len(sur_k)):
            rejected.append(b)
            continue
        for which, x in enumerate((sur_k[merge_row[b]], sur_v[merge_row[b]]) if k else (new_k[b], new_v[b])):
            c, s = quantise(x)
            codes[:, page, which, :, slot % page_size] = c
            scale_codes[:, page, which, :, slot % page_size] = s
        n = slot + 1
        if -(-n // page_size) < -(-(L + 1) // page_size):
            released[b] = row[-(-n // page_size)]
            row[-(-n // page_size)] = -1
        bt[b], lens[b] = row, n
    return codes, scale_codes, bt, lens, released, rejected
