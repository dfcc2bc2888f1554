"""The 8-bit paged cache and attention over shared prefixes, as timed cases.

Kinds of cases:

  write   rows of K and V quantised into the pages of one layer (prompts, or one row a sequence)
  append  one entry for every sequence in all layers, quantised; some complete a merge
  read    entries of the 8-bit cache back as packed bf16 rows
  attend  decode attention over the 8-bit cache
  shared  decode attention of groups of sequences that share a prefix, over a 16- or an 8-bit cache

The 8-bit cache holds e4m3 values [layers][pages][2][heads][16][D] and a power of two for each row of D
[layers][pages][2][heads][16]: the smallest 2^e with which the row's largest magnitude is at most 448 * 2^e.
K rows have a few large channels, as keys after a rotary embedding do.
"""
import math

import torch

own = False

PAGE = 16


def listed():
    return [
        # the prompts of a prefill batch of 16 x ~2048 tokens, K and V inside fused projection rows
        dict(name="prompt write", kind="write", B=16, T=32768, Hkv=8, D=128, fused=True, single=False),
        # one layer's new tokens of a decode step: latency
        dict(name="token write", kind="write", B=48, T=48, Hkv=8, D=128, fused=True, single=True),
        # a decode step's entries of a 32-layer model, one in ten sequences merging
        dict(name="append 32 layers", kind="append", B=64, layers=32, Hkv=8, D=128, merges=0.1),
        # the smallest: one sequence of a small model
        dict(name="append small", kind="append", B=1, layers=4, Hkv=2, D=64, merges=0.0),
        # cached prompts read back for a prefill that goes on behind them
        dict(name="prompt read", kind="read", B=4, T=65536, Hkv=8, D=128, fused=False, single=False),
        # short odd prompts of a small head
        dict(name="odd read", kind="read", B=7, T=2501, Hkv=5, D=64, fused=False, single=False),
        # one short conversation: latency
        dict(name="short attention", kind="attend", B=1, T=421, Hq=8, Hkv=2, D=64),
        # a serving batch of 64 sequences of about 1200 entries, ragged
        dict(name="serving attention", kind="attend", B=64, T=76800, Hq=32, Hkv=8, D=128),
        # four long contexts, seven query heads a KV head
        dict(name="long attention", kind="attend", B=4, T=131072, Hq=28, Hkv=4, D=128),
        # eight samples of one prompt, a few hundred tokens in
        dict(name="samples", kind="shared", n=1, B=8, P=4099, T=1700, Hq=32, Hkv=8, D=128, bits=16),
        # a chat batch behind one long system prompt
        dict(name="system prompt", kind="shared", n=1, B=64, P=16384, T=16384, Hq=32, Hkv=8, D=128, bits=16),
        # five long documents with 24 questions each, over the 8-bit cache
        dict(name="documents", kind="shared", n=5, B=120, P=12007, T=9600, Hq=32, Hkv=8, D=128, bits=8),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["write", "append", "read", "attend", "attend", "shared", "shared", "shared"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 3, 4, 8, 8])
    if kind in ("write", "read"):
        single = rng.random() < 0.3
        B = _log_int(rng, 1, 256)
        T = B if single else max(B, _log_int(rng, 40, 32768))
        return dict(kind=kind, B=B, T=T, Hkv=Hkv, D=D, fused=rng.random() < 0.5, single=single)
    if kind == "append":
        return dict(kind=kind, B=_log_int(rng, 1, 64), layers=rng.randrange(1, 33), Hkv=Hkv, D=D, merges=rng.choice([0.0, 0.1, 0.3]))
    G = rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
    if kind == "attend":
        B = _log_int(rng, 1, 128)
        return dict(kind=kind, B=B, T=max(B, _log_int(rng, 100, 131072)), Hq=G * Hkv, Hkv=Hkv, D=D)
    n = rng.choice([1, 1, 1, 2, 3, 5])
    B = max(n, _log_int(rng, 2, 96))
    P = _log_int(rng, 100, 16384 // n)
    return dict(kind=kind, n=n, B=B, P=P, T=_log_int(rng, B, 16384), Hq=G * Hkv, Hkv=Hkv, D=D, bits=rng.choice([16, 8]))


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
class _Draw:
    def __init__(self, seed):
        self.dev = torch.device("cuda")
        self.gen = torch.Generator(device=self.dev)
        self.gen.manual_seed(seed)
        self.host = torch.Generator()
        self.host.manual_seed(seed)

    def rows(self, *shape):
        """bf16 rows [..][heads][D], every eleventh channel six times as large."""
        x = torch.randn(shape, generator=self.gen, device=self.dev)
        x[..., 3::11] *= 6.0
        return x.bfloat16()

    def split(self, total, n, least):
        """n lengths of at least `least` that add up to total."""
        w = torch.exp(0.7 * torch.randn(n, generator=self.host, dtype=torch.float64))
        cut = (torch.cumsum(w, 0) / w.sum() * (total - least * n)).long()
        cut[-1] = total - least * n
        return torch.diff(cut, prepend=torch.zeros(1, dtype=torch.long)) + least

    def tables(self, lens, columns=None, total=None):
        """(block table [n][columns], by default as many as there have to be, of pages of a pool of `total` in any order
        and -1 behind a sequence's last; total)."""
        pages = (lens + PAGE - 1) // PAGE
        columns, total, used = columns or max(1, int(pages.max())), total or int(pages.sum()), int(pages.sum())
        table = torch.full((lens.numel(), columns), -1, dtype=torch.int32)
        table[torch.arange(columns)[None] < pages[:, None]] = torch.randperm(total, generator=self.host)[:used].int()
        return table, total

    def ints(self, lo, hi, n):
        return torch.randint(lo, hi, (n,), generator=self.host)


def _pages_of(rows_k, rows_v):
    """[layers][pages][2][heads][16][D] out of rows [layers][pages][16][heads][D]."""
    return torch.stack([rows_k, rows_v], 2).transpose(3, 4).contiguous()


def prepare(case, seed):
    d, s, kind = _Draw(seed), dict(case), case["kind"]
    dev, Hkv, D = d.dev, case["Hkv"], case["D"]
    if kind in ("write", "read"):
        B, T = case["B"], case["T"]
        rows = torch.ones(B, dtype=torch.long) if case["single"] else d.split(T, B, 0)
        before = 300 if case["single"] else 40   # entries that a sequence holds already, at most
        start = d.ints(0, before, B)
        table, pages = d.tables(start + rows, total=T // PAGE + B * (before // PAGE + 2))
        s["bt"], s["start"] = table.to(dev), start.int().to(dev)
        s["cu"] = None if case["single"] else torch.cat([torch.zeros(1, dtype=torch.long), rows.cumsum(0)]).int().to(dev)
        at = torch.repeat_interleave(torch.arange(B), rows)
        entry = torch.arange(T) - (rows.cumsum(0) - rows)[at] + start[at]
        s["page"], s["slot"] = table[at, entry // PAGE].long().to(dev), (entry % PAGE).to(dev)
        if kind == "write":
            s["values"] = torch.zeros((1, pages, 2, Hkv, PAGE, D), device=dev).to(torch.float8_e4m3fn)
            s["scales"] = torch.full((1, pages, 2, Hkv, PAGE), 127, dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu)
            x = d.rows(T, 2 * Hkv, D)
            if case["fused"]:   # the rows of a projection, whose first third would be queries
                x = torch.cat([torch.zeros_like(x[:, :Hkv]), x], 1)
            s["k"], s["v"] = x[:, -2 * Hkv:-Hkv], x[:, -Hkv:]
            if not case["fused"]:
                s["k"], s["v"] = s["k"].contiguous(), s["v"].contiguous()
        else:
            s["values"], s["scales"] = _quantise(_pages_of(*d.rows(2, 1, pages, PAGE, Hkv, D)))
        return s
    if kind == "append":
        B, layers = case["B"], case["layers"]
        lens = d.ints(3, 56, B)
        table, pages = d.tables(lens, columns=5, total=4 * B)
        s["state0"] = torch.cat([lens.int(), table.reshape(-1)]).to(dev)
        s["state"] = s["state0"].clone()
        s["lens"], s["bt"] = s["state"][:B], s["state"][B:].view(B, -1)
        s["new_pages"] = (pages + torch.arange(B)).int().to(dev)
        k = torch.where(torch.rand(B, generator=d.host) < case["merges"], d.ints(2, 4, B), 0)
        s["merge_k"] = k.int().to(dev)
        s["merge_row"] = (torch.where(k > 0, (k > 0).cumsum(0) - 1, 0)).int().to(dev)
        n = max(1, int((k > 0).sum()))
        s["new"], s["surrogate"] = d.rows(2, B, layers, Hkv, D), d.rows(2, n, layers, Hkv, D)
        s["values"] = torch.zeros((layers, pages + B, 2, Hkv, PAGE, D), device=dev).to(torch.float8_e4m3fn)
        s["scales"] = torch.full((layers, pages + B, 2, Hkv, PAGE), 127, dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu)
        return s
    B = case["B"]
    lens = d.split(case["T"], B, 0)
    prefixes = torch.tensor(_prefix_lens(case) if kind == "shared" else [], dtype=torch.long)
    table, pages = d.tables(torch.cat([lens, prefixes]))
    pool = _pages_of(*d.rows(2, 1, pages, PAGE, Hkv, D))
    s["q"] = torch.randn((B, case["Hq"], D), generator=d.gen, device=dev).bfloat16()
    s["bt"], s["lens"] = table[:B].contiguous().to(dev), lens.int().to(dev)
    if kind == "shared":
        s["prefix_bt"], s["prefix_lens"] = table[B:].contiguous().to(dev), prefixes.int().to(dev)
        sizes = d.split(B, case["n"], 1)
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.long), sizes.cumsum(0)]).int().to(dev)
        s["most"] = int(sizes.max())
    if case.get("bits", 8) == 16:
        s["pool"] = pool
    else:
        s["values"], s["scales"] = _quantise(pool)
    return s


def _prefix_lens(case):
    return [max(1, case["P"] - 37 * i) for i in range(case["n"])]


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if kind == "append":
        s["state"].copy_(s["state0"])   # the lengths and tables before the step
    if own:
        import paper_2609_27233_gb300 as umim
        if "pool" not in s:
            pool = umim.Kv8Pool(s["values"], s["scales"])
        if kind == "write":
            umim.umim_kv8_write(pool, 0, s["bt"], s["start"], s["k"], s["v"], cu_rows=s["cu"])
            return dict(values=s["values"], scales=s["scales"])
        if kind == "read":
            return umim.umim_kv8_read(pool, 0, s["bt"], s["start"], s["T"], cu_rows=s["cu"])
        if kind == "append":
            released = umim.umim_kv8_append_merge(
                pool, s["bt"], s["lens"], s["new"][0], s["new"][1], s["new_pages"], s["merge_k"], s["merge_row"],
                s["surrogate"][0], s["surrogate"][1])
            return dict(values=s["values"], scales=s["scales"], lens=s["lens"], bt=s["bt"], released=released)
        if kind == "attend":
            if "ws" not in s:
                s["ws"] = umim.workspace(umim.umim_decode_attention_kv8_workspace_size(
                    s["B"], s["Hq"], s["Hkv"], s["D"]), s["q"].device)
            return umim.umim_decode_attention_kv8(s["q"], pool, 0, s["bt"], s["lens"], workspace_buf=s["ws"])
        if "ws" not in s:
            s["ws"] = umim.workspace(umim.umim_decode_attention_shared_workspace_size(
                s["B"], s["n"], s["Hq"], s["Hkv"], s["D"]), s["q"].device)
        if s["bits"] == 16:
            return umim.umim_decode_attention_shared(
                s["q"], s["pool"], 0, s["prefix_bt"], s["prefix_lens"], s["bt"], s["lens"], prefix_offsets=s["offsets"],
                workspace_buf=s["ws"])
        return umim.umim_decode_attention_shared_kv8(
            s["q"], pool, 0, s["prefix_bt"], s["prefix_lens"], s["bt"], s["lens"], prefix_offsets=s["offsets"],
            workspace_buf=s["ws"])
    if kind == "write":
        x = torch.stack([s["k"], s["v"]], 1)
        values, scales = _quantise(x)
        s["values"].view(torch.uint8)[0, s["page"], :, :, s["slot"]] = values.view(torch.uint8)
        s["scales"].view(torch.uint8)[0, s["page"], :, :, s["slot"]] = scales.view(torch.uint8)
        return dict(values=s["values"], scales=s["scales"])
    if kind == "read":
        values = s["values"].view(torch.uint8)[0, s["page"], :, :, s["slot"]].view(torch.float8_e4m3fn).float()
        scales = s["scales"].view(torch.uint8)[0, s["page"], :, :, s["slot"]].int() - 127
        k, v = (values * _power(scales)[..., None]).bfloat16().unbind(1)
        return k.contiguous(), v.contiguous()
    if kind == "append":
        return _append_merge(s)
    if kind == "attend":
        k, v = _entries(s, s["bt"])
        return _attention([(s["q"], k, v, s["lens"], None)])
    k, v = _entries(s, s["bt"])
    pk, pv = _entries(s, s["prefix_bt"])
    group = torch.searchsorted(s["offsets"], torch.arange(s["B"], device=s["q"].device), right=True) - 1
    place = torch.arange(s["B"], device=s["q"].device) - s["offsets"][group]
    return _attention([(s["q"], k, v, s["lens"], None), (s["q"], pk, pv, s["prefix_lens"], (group, place, s["most"]))])


def _power(e):
    """2^e in fp32."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """(e4m3 values, powers of two) of the rows of x."""
    x = x.float()
    fraction, power = torch.frexp(x.abs().amax(-1))   # largest = fraction * 2^power, fraction in [0.5, 1)
    e = (power - 9 + (fraction > 0.875)).clamp(-100, 120)
    e = torch.where(fraction > 0, e, 0)
    return (x * _power(-e)[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _append_merge(s):
    lens, bt, k = s["lens"].long(), s["bt"], s["merge_k"].long()
    B, row = lens.numel(), torch.arange(lens.numel(), device=lens.device)
    opens = lens % PAGE == 0
    column = lens // PAGE
    bt[row, column] = torch.where(opens, s["new_pages"], bt[row, column])
    slot = torch.where(k > 0, lens + 1 - k, lens)
    page = bt[row, slot // PAGE].long()
    x = torch.where((k > 0)[None, :, None, None, None], s["surrogate"][:, s["merge_row"].long()], s["new"])
    values, scales = _quantise(x.permute(1, 2, 0, 3, 4))   # [B][layers][2][heads][D]
    s["values"].view(torch.uint8)[:, page, :, :, slot % PAGE] = values.view(torch.uint8)
    s["scales"].view(torch.uint8)[:, page, :, :, slot % PAGE] = scales.view(torch.uint8)
    after = torch.where(k > 0, slot, lens) + 1
    drops = (after + PAGE - 1) // PAGE < column + 1
    released = torch.where(drops, bt[row, column], -1)
    bt[row, column] = torch.where(drops, -1, bt[row, column])
    s["lens"].copy_(after)
    return dict(values=s["values"], scales=s["scales"], lens=s["lens"], bt=bt, released=released)


def _entries(s, table):
    """K and V in fp32 [sequences][entries][heads][D] of the pages in a table."""
    at = table.long().clamp_min(0)
    if "pool" in s:
        x = s["pool"][0, at].float()
    else:
        x = s["values"].view(torch.uint8)[0, at].view(torch.float8_e4m3fn).float()
        x = x * _power(s["scales"].view(torch.uint8)[0, at].int() - 127)[..., None]
    return x.permute(2, 0, 1, 4, 3, 5).flatten(2, 3).unbind(0)   # [2][n][pages][16][heads][D]


def _attention(parts):
    """Softmax attention of every query over the entries of all parts; a part of groups holds one set of entries a group."""
    q = parts[0][0]
    B, Hq, D = q.shape
    scores, held = [], []
    for q, k, v, lens, groups in parts:
        Hkv = k.shape[2]
        x = q.float().view(B, Hkv, Hq // Hkv, D) / math.sqrt(D)
        if groups is not None:
            group, place, most = groups
            x = torch.zeros((k.shape[0], most) + x.shape[1:], device=x.device).index_put_((group, place), x)
            y = torch.einsum("npgjd,nlgd->npgjl", x, k)
            y = y.masked_fill((torch.arange(k.shape[1], device=x.device) >= lens[:, None])[:, None, None, None], -math.inf)
            scores.append(y[group, place])
        else:
            y = torch.einsum("bgjd,blgd->bgjl", x, k)
            scores.append(y.masked_fill((torch.arange(k.shape[1], device=x.device) >= lens[:, None])[:, None, None], -math.inf))
        held.append((v, groups))
    m = torch.stack([y.amax(-1) for y in scores]).amax(0).clamp_min(-1e30)[..., None]
    total, out = 0.0, 0.0
    for y, (v, groups) in zip(scores, held):
        p = (y - m).exp()
        total = total + p.sum(-1, keepdim=True)
        if groups is not None:
            group, place, most = groups
            p = torch.zeros((v.shape[0], most) + p.shape[1:], device=p.device).index_put_((group, place), p)
            out = out + torch.einsum("npgjl,nlgd->npgjd", p, v)[group, place]
        else:
            out = out + torch.einsum("bgjl,blgd->bgjd", p, v)
    return (out / torch.where(total > 0, total, 1.0)).reshape(B, Hq, D).bfloat16()


# ----------------------------------------------------------------------------
# what a pass cannot do without, and what it returns in 64 bits
# ----------------------------------------------------------------------------
def work(case):
    Hkv, D, kind = case["Hkv"], case["D"], case["kind"]
    wide, narrow = 4 * Hkv * D, 2 * Hkv * (D + 1)   # bytes of an entry's K and V in one layer
    if kind in ("write", "read"):
        return dict(bytes=case["T"] * (wide + narrow), flops=4.0 * case["T"] * Hkv * D)
    if kind == "append":
        n = case["B"] * case["layers"]
        return dict(bytes=n * (wide + narrow), flops=4.0 * n * Hkv * D)
    each = wide if case.get("bits", 8) == 16 else narrow
    prefixes = _prefix_lens(case) if kind == "shared" else []
    ends = 4 * case["B"] * case["Hq"] * D
    pairs = case["T"] + (case["B"] * sum(prefixes) / case["n"] if prefixes else 0)
    return dict(bytes=(case["T"] + sum(prefixes)) * each + ends, flops=4.0 * case["Hq"] * D * pairs)


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "read":
        x = _values64(s)[0, s["page"], :, :, s["slot"]]
        return x[:, 0].contiguous(), x[:, 1].contiguous()
    if kind == "write":
        values, scales = s["values"].double(), torch.full(s["scales"].shape, 1.0, dtype=torch.float64, device=s["k"].device)
        for which, x in enumerate((s["k"], s["v"])):
            c, r = _round_e4m3(x.double())
            values[0, s["page"], which, :, s["slot"]] = c
            scales[0, s["page"], which, :, s["slot"]] = r
        return dict(values=values, scales=scales)
    if kind == "append":
        lens, bt, k = s["lens"].tolist(), s["bt"].clone(), s["merge_k"].tolist()
        values, scales = s["values"].double(), torch.full(s["scales"].shape, 1.0, dtype=torch.float64, device=bt.device)
        for b, length in enumerate(lens):
            source = s["surrogate"][:, int(s["merge_row"][b])] if k[b] else s["new"][:, b]
            slot = length + 1 - k[b] if k[b] else length
            page = int(s["new_pages"][b]) if slot == length and length % PAGE == 0 else int(bt[b, slot // PAGE])
            for which in range(2):
                c, r = _round_e4m3(source[which].double())
                values[:, page, which, :, slot % PAGE] = c
                scales[:, page, which, :, slot % PAGE] = r
        return dict(values=values, scales=scales, lens=None, bt=None, released=None)
    q, (B, Hq, D), Hkv = s["q"].double(), s["q"].shape, case["Hkv"]
    pool = s["pool"].double() if "pool" in s else _values64(s)
    offsets = s["offsets"].tolist() if kind == "shared" else []
    out = torch.zeros((B, Hq, D), dtype=torch.float64, device=q.device)
    for b in range(B):
        tables = [(s["bt"][b], int(s["lens"][b]))]
        if kind == "shared":
            g = max(i for i in range(case["n"]) if offsets[i] <= b)
            tables.append((s["prefix_bt"][g], int(s["prefix_lens"][g])))
        rows = torch.cat([pool[0, t[:-(-n // PAGE)].long()].permute(1, 0, 3, 2, 4).flatten(1, 2)[:, :n] for t, n in tables], 1)
        if rows.shape[1]:
            k, v = rows.repeat_interleave(Hq // Hkv, 2).unbind(0)
            w = torch.softmax((k * q[b]).sum(-1) / math.sqrt(D), 0)
            out[b] = (w[..., None] * v).sum(0)
    return out


def _values64(s):
    return s["values"].double() * _power64(s["scales"].view(torch.uint8).long() - 127)[..., None]


def _power64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _round_e4m3(x):
    """(the nearest e4m3 numbers, ties to even, of x / 2^e, the rows' 2^e), e the smallest with |x| <= 448 * 2^e."""
    most = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2((most / 448).clamp_min(1e-300)))
    e = e.clamp(-100, 120)
    e = torch.where(448 * _power64(e - 1) >= most, e - 1, e)   # where the logarithm was rounded over a whole number
    e = torch.where(448 * _power64(e) < most, e + 1, e).clamp(-100, 120)
    e = torch.where(most > 0, e, 0.0)
    y = x / _power64(e)
    size = torch.frexp(y.abs().clamp_min(2.0 ** -6))[1]   # magnitudes in [2^(size - 1), 2^size) are 2^(size - 4) apart
    step = _power64(size - 4)
    return torch.round(y / step) * step, _power64(e)[..., 0]
