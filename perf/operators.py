"""Log probabilities, their gradient, and distillation from a teacher's top logits, as timed cases.

Kinds of cases:

  logprobs  log probabilities of given tokens, entropy and the best alternatives over [rows][vocab] logits
  grad      the gradient of those log probabilities and entropies with respect to the logits
  topk      soft-target cross-entropy from a teacher's cached top log probabilities and its gradient

Logits are N(0, 2^2) with 50 tokens a row raised by an exponential draw, so that a row has a few likely
tokens and a long tail, as a language model's rows do.  A share `masked` of the rows allows 12 tokens only (the
others are -inf, as a grammar does it); a share `left_out` of the rows has no token (-1: padding).
"""
import math

import torch

own = False

VOCAB = 128256
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # one chat request that asks for log probabilities: the new token's row, 20 alternatives
        dict(name="one row", kind="logprobs", R=1, V=VOCAB, dtype="bf16", T=1.0, n_top=20, masked=0.0, left_out=0.0),
        # a decode step of 128 sequences, some under a grammar, 5 alternatives each
        dict(name="decode batch", kind="logprobs", R=128, V=VOCAB, dtype="bf16", T=0.7, n_top=5, masked=0.1,
             left_out=0.0),
        # scoring packed prompts (perplexity): tokens only, some rows padding
        dict(name="scored prompts", kind="logprobs", R=8192, V=VOCAB, dtype="bf16", T=1.0, n_top=0, masked=0.0,
             left_out=0.02),
        # the teacher's top-64 cache of a training batch of 8 x 512 tokens
        dict(name="teacher cache", kind="logprobs", R=4096, V=VOCAB, dtype="bf16", T=1.0, n_top=64, masked=0.0,
             left_out=0.0),
        # fp32 logits over a vocabulary that fills no vector
        dict(name="odd vocabulary", kind="logprobs", R=333, V=50257, dtype="fp32", T=1.3, n_top=10, masked=0.05,
             left_out=0.1),
        # hard labels and an entropy term on a batch of 8 x 512 tokens
        dict(name="label gradient", kind="grad", R=4096, V=VOCAB, dtype="bf16", T=1.0, entropy=True, left_out=0.1),
        # a small model's short batch in fp32, labels only
        dict(name="small gradient", kind="grad", R=45, V=32000, dtype="fp32", T=1.0, entropy=False, left_out=0.0),
        # the distillation objective on 8 x 512 tokens from a top-64 cache
        dict(name="top-64 batch", kind="topk", R=3260, N=2870, V=VOCAB, K=64, dtype="bf16", T=1.0, tail=True),
        # the same on a large batch with the top 20 renormalised
        dict(name="top-20 large", kind="topk", R=9600, N=8700, V=VOCAB, K=20, dtype="bf16", T=2.0, tail=False),
        # a short sample's few pairs: latency
        dict(name="few pairs", kind="topk", R=21, N=17, V=VOCAB, K=50, dtype="bf16", T=1.0, tail=True),
        # a small vocabulary of odd size in fp16, the longest lists
        dict(name="fp16 odd", kind="topk", R=700, N=611, V=50257, K=128, dtype="fp16", T=1.0, tail=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["logprobs", "logprobs", "grad", "topk", "topk"])
    V = rng.choice([32000, 50257, VOCAB, VOCAB, 151936, rng.randrange(2000, VOCAB)])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    T = round(rng.uniform(0.5, 2.0), 2)
    most = 4096 * VOCAB // V // (2 if dtype == "fp32" else 1)
    R = _log_int(rng, 1, most)
    if kind == "logprobs":
        return dict(kind=kind, R=R, V=V, dtype=dtype, T=T, n_top=rng.choice([0, rng.randrange(1, 129), rng.randrange(1, 33)]),
                    masked=rng.choice([0.0, 0.1]), left_out=rng.choice([0.0, 0.2]))
    if kind == "grad":
        return dict(kind=kind, R=R, V=V, dtype=dtype, T=T, entropy=rng.random() < 0.5, left_out=rng.choice([0.0, 0.2]))
    return dict(kind=kind, R=R, N=max(1, int(R * rng.uniform(0.5, 1.0))), V=V, K=rng.randrange(1, 129), dtype=dtype, T=T,
                tail=rng.random() < 0.6)


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
class _Draw:
    def __init__(self, seed):
        self.dev = torch.device("cuda")
        self.gen = torch.Generator(device=self.dev)
        self.gen.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device=self.dev)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.gen, device=self.dev)

    def ints(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.gen, device=self.dev)

    def distinct(self, R, n, V):
        """[R][n] ids, distinct within a row: an arithmetic progression modulo V that does not wrap round."""
        step = 1 + (self.uniform(R, 1) * max(1, (V - 1) // n)).long().clamp(max=max(0, (V - 1) // n - 1))
        return (self.ints(0, V, R, 1) + step * torch.arange(n, device=self.dev)) % V

    def logits(self, R, V, dtype):
        """[R][ld] in blocks of rows, and the raised ids [R][n]."""
        ld = -(-V // 8) * 8
        out = torch.empty((R, ld), dtype=dtype, device=self.dev)
        ids = self.distinct(R, min(50, V), V)
        up = -3.0 * torch.log(self.uniform(*ids.shape).clamp_min(1e-6))
        for r in range(0, R, 1024):
            x = self.normal(min(1024, R - r), ld).mul_(2.0)
            out[r:r + 1024] = x.scatter_add_(1, ids[r:r + 1024], up[r:r + 1024])
        return out, ids


def prepare(case, seed):
    d, V, R = _Draw(seed), case["V"], case["R"]
    x, ids = d.logits(R, V, DTYPES[case["dtype"]])
    s = dict(case, x=x)
    if case["kind"] in ("logprobs", "grad"):
        near = ids.gather(1, d.ints(0, ids.shape[1], R, 1))[:, 0]
        tok = torch.where(d.uniform(R) < 0.7, near, d.ints(0, V, R))
        s["tokens"] = torch.where(d.uniform(R) < case["left_out"], -1, tok).int()
    if case["kind"] == "logprobs":
        rows = (d.uniform(R) < case["masked"]).nonzero()[:, 0]
        if rows.numel():
            allowed = d.distinct(rows.numel(), min(12, V), V)
            held = x[rows].gather(1, allowed)
            x[rows] = torch.full((1, 1), -math.inf, dtype=x.dtype, device=x.device).expand(rows.numel(), x.shape[1]).scatter(1, allowed, held)
    if case["kind"] == "grad":   # what the forward pass has left
        m, l, h = _statistics(x[:, :V], case["T"])
        left = s["tokens"] < 0
        s["stats"] = torch.stack([m, l], 1).masked_fill_(left[:, None], 0.0)
        s["entropy_of"] = h.masked_fill_(left, 0.0)
        s["g"] = -(0.5 + d.uniform(R)) / R
        s["h"] = -0.01 * (0.5 + d.uniform(R)) / R if case["entropy"] else None
    if case["kind"] == "topk":
        K, N, R_T = case["K"], case["N"], case["N"] + case["N"] // 4 + 1
        top = d.distinct(R_T, min(K, V), V)
        w = (3.0 * d.normal(*top.shape)).sort(dim=1, descending=True)[0]
        mass = 0.6 + 0.39 * d.uniform(R_T, 1)
        s["top_logprobs"] = (w - w.logsumexp(1, keepdim=True) + mass.log()).contiguous()
        s["top_ids"] = top.int().contiguous()
        s["top_ids"][:, K - K // 8:][d.uniform(R_T) < 0.1] = -1   # rows whose teacher had fewer alternatives
        s["t_rows"] = torch.randperm(R_T, generator=d.gen, device=d.dev)[:N].sort()[0].int()
        s["s_rows"] = torch.randperm(R, generator=d.gen, device=d.dev)[:N].sort()[0].int()
        # the student's rows lie near the teacher's
        at, sr = top[s["t_rows"].long()], s["s_rows"].long()
        near = case["T"] * (s["top_logprobs"][s["t_rows"].long()] + 14.0 + 0.5 * d.normal(N, top.shape[1]))
        for r in range(0, N, 1024):
            rows = sr[r:r + 1024]
            x[rows] = x[rows].scatter(1, at[r:r + 1024], near[r:r + 1024].to(x.dtype))
        s["n"] = torch.tensor([N], dtype=torch.int32, device=d.dev)
    return s


def _statistics(x, T):
    """(row maximum, ln of the sum of exp((x - maximum) / T), entropy), in blocks of rows."""
    m = torch.empty(x.shape[0], device=x.device)
    l, h = torch.empty_like(m), torch.empty_like(m)
    for r in range(0, x.shape[0], 512):
        b = x[r:r + 512].double()
        m[r:r + 512] = b.amax(1)
        y = (b - b.amax(1, keepdim=True)) / T
        z = y.logsumexp(1, keepdim=True)
        l[r:r + 512], h[r:r + 512] = z[:, 0], -((y - z).exp() * (y - z)).sum(1)
    return m, l, h


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------
def run(s):
    if own:
        import paper_2609_27233_gb300 as umim
        V = s["V"]
        if s["kind"] == "logprobs":
            return umim.umim_token_logprobs(s["x"], s["tokens"], n_top=s["n_top"], vocab=V, temperature=s["T"])
        if s["kind"] == "grad":
            return umim.umim_token_logprobs_grad(s["x"], s["stats"], s["tokens"], s["g"], s["entropy_of"], s["h"], vocab=V,
                                                 temperature=s["T"])[:, :V]
        if "ws" not in s:
            s["ws"] = umim.workspace(umim.umim_distill_topk_ce_workspace_size(s["R"], s["N"]), s["x"].device)
        loss, pair_loss, grad = umim.umim_distill_topk_ce(
            s["top_ids"], s["top_logprobs"], s["x"], s["t_rows"], s["s_rows"], n_pairs=s["n"], vocab=V,
            temperature=s["T"], tail=s["tail"], workspace_buf=s["ws"])
        return loss, pair_loss, grad[:, :V]
    if s["kind"] == "logprobs":
        return _logprobs(s["x"][:, :s["V"]], s["tokens"].long(), s["T"], s["n_top"])
    if s["kind"] == "grad":
        return _logprobs_grad(s["x"][:, :s["V"]], s["stats"], s["tokens"].long(), s["g"], s["entropy_of"], s["h"], s["T"])
    return _topk_ce(s["top_ids"], s["top_logprobs"], s["x"][:, :s["V"]], s["t_rows"].long(), s["s_rows"].long(), s["T"],
                    s["tail"])


def _logprobs(x, tokens, T, n_top):
    left = tokens < 0
    x = x.float()
    m = x.amax(1)
    y = (x - m[:, None]) / T
    e = y.exp()
    total = e.sum(1)
    l = total.log()
    out = dict(logprobs=(y.gather(1, tokens.clamp_min(0)[:, None])[:, 0] - l).masked_fill_(left, 0.0),
               entropy=(l - torch.where(e > 0, e * y, 0.0).sum(1) / total).masked_fill_(left, 0.0),
               stats=torch.stack([m, l], 1).masked_fill_(left[:, None], 0.0))
    if n_top:
        best, ids = x.sort(dim=1, descending=True, stable=True)
        best, ids = best[:, :n_top], ids[:, :n_top]
        none = left[:, None] | (best == -math.inf)
        out["top_ids"] = ids.masked_fill(none, -1).int()
        out["top_logprobs"] = ((best - m[:, None]) / T - l[:, None]).masked_fill_(none, -math.inf)
    return out


def _logprobs_grad(x, stats, tokens, g, entropy, h, T):
    left = tokens < 0
    z = (x.float() - stats[:, :1]) / T - stats[:, 1:]
    p = z.exp()
    at = tokens.clamp_min(0)[:, None]
    z_t = z.gather(1, at)
    d = -g[:, None] * p
    d.scatter_(1, at, -g[:, None] * torch.expm1(z_t))
    if h is not None:
        d -= h[:, None] * torch.where(p > 0, p * (z + entropy[:, None]), 0.0)
    return (d / T).masked_fill_(left[:, None], 0.0).to(x.dtype)


def _topk_ce(top_ids, top_logprobs, student, t_rows, s_rows, T, tail):
    N, V = t_rows.numel(), student.shape[1]
    x = student[s_rows].float()
    ids, held = top_ids[t_rows].long(), top_ids[t_rows] >= 0
    lt = top_logprobs[t_rows].double().masked_fill_(~held, -math.inf)
    if tail:
        p = lt.exp()
        rest = (1.0 - p.sum(1)).clamp_min(0.0)
    else:
        p = (lt - lt.amax(1, keepdim=True)).exp()
        p = p / p.sum(1, keepdim=True)
        rest = torch.zeros_like(p[:, 0])
    p, rest = p.float(), rest.float()
    inside = torch.zeros((N, V + 1), dtype=torch.bool, device=x.device).scatter_(1, ids.where(held, V), True)[:, :V]
    y = (x - x.amax(1, keepdim=True)) / T
    e = y.exp()
    z_rest = e.masked_fill(inside, 0.0).sum(1)
    at = ids.clamp_min(0)
    z = z_rest + (y.gather(1, at).exp() * held).sum(1)
    log_q = y.gather(1, at) - z.log()[:, None]
    pair_loss = -torch.where(p > 0, p * log_q, 0.0).sum(1) - torch.where(rest > 0, rest * (z_rest / z).log(), 0.0)
    whole = p.sum(1) + rest
    outside = torch.where(rest > 0, whole - rest * z / z_rest, whole)
    d = (e / z[:, None]) * torch.where(inside, whole[:, None], outside[:, None])
    d.scatter_add_(1, at, -p * held)
    grad = torch.zeros_like(student)
    grad[s_rows] = (d / (N * T)).to(student.dtype)
    return pair_loss.double().mean().float().reshape(1), pair_loss, grad


# ----------------------------------------------------------------------------
# what a pass cannot do without, and what it returns in 64 bits
# ----------------------------------------------------------------------------
def work(case):
    R, V, w = case["R"], case["V"], 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "logprobs":
        kept = R * (1.0 - case["left_out"])
        return dict(bytes=kept * V * w + R * (4 + 16 + 8 * case["n_top"]), flops=6.0 * kept * V)
    if case["kind"] == "grad":
        kept = R * (1.0 - case["left_out"])
        return dict(bytes=(kept + R) * V * w + R * 24, flops=(8.0 if case["entropy"] else 5.0) * kept * V)
    N, K = case["N"], case["K"]
    return dict(bytes=(N + R) * V * w + N * (8 * K + 12), flops=8.0 * N * V)


def exact(case, seed):
    s = prepare(case, seed)
    V, T, parts = s["V"], s["T"], []
    if s["kind"] == "topk":
        return _exact_topk(s)
    for r in range(0, s["R"], 256):
        x, t = s["x"][r:r + 256, :V], s["tokens"][r:r + 256].long()
        left, logp = t < 0, torch.log_softmax(x.double() / T, 1)
        p = logp.exp()
        plogp = (p * logp).nan_to_num_(nan=0.0)
        lp_t = logp[torch.arange(len(t), device=t.device), t.clamp_min(0)]
        if s["kind"] == "grad":
            one = torch.nn.functional.one_hot(t.clamp_min(0), V)
            d = s["g"][r:r + 256, None].double() * (one - p)
            if s["h"] is not None:
                d -= s["h"][r:r + 256, None].double() * (plogp - p * plogp.sum(1, keepdim=True))
            parts.append((d / T).masked_fill_(left[:, None], 0.0).float())
            continue
        best = x.double().max(1)[0]
        stats = torch.stack([best, torch.logsumexp(x.double() / T, 1) - best / T], 1)
        got = dict(logprobs=lp_t.masked_fill(left, 0.0), entropy=(-plogp.sum(1)).masked_fill(left, 0.0),
                   stats=stats.masked_fill(left[:, None], 0.0))
        if s["n_top"]:
            # a key for each logit whose order is that of (value, lowest id first)
            b = (x.float() + 0.0).view(torch.int32).long()
            key = torch.where(b < 0, b ^ 0x7fffffff, b) * (1 << 20) + (V - 1 - torch.arange(V, device=x.device))
            at = V - 1 - (key.topk(s["n_top"], 1)[0] & ((1 << 20) - 1))
            none = left[:, None] | (x.gather(1, at) == -math.inf)
            got["top_ids"] = at.masked_fill(none, -1).int()
            got["top_logprobs"] = logp.gather(1, at).masked_fill(none, -math.inf)
        parts.append(got)
    if s["kind"] == "grad":
        return torch.cat(parts)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_topk(s):
    V, T, N = s["V"], s["T"], s["N"]
    grad, losses = torch.zeros((s["R"], V), dtype=torch.float32, device=s["x"].device), []
    for r in range(0, N, 256):
        tr, sr = s["t_rows"][r:r + 256].long(), s["s_rows"][r:r + 256].long()
        logq = torch.log_softmax(s["x"][sr, :V].double() / T, 1)
        n, dev = len(sr), logq.device
        ids = s["top_ids"][tr].long()
        w = torch.where(ids >= 0, s["top_logprobs"][tr].double().exp(), 0.0)
        if not s["tail"]:
            w = w / w.sum(1, keepdim=True)
        target = torch.zeros((n, V + 1), dtype=torch.float64, device=dev)
        inside = torch.zeros((n, V + 1), dtype=torch.bool, device=dev)
        slot = torch.where(ids >= 0, ids, V)
        target.scatter_add_(1, slot, w)
        inside.scatter_(1, slot, True)
        target, inside = target[:, :V], inside[:, :V]
        rest = (1.0 - target.sum(1, keepdim=True)).clamp_min(0.0) if s["tail"] else torch.zeros((n, 1), device=dev).double()
        q = logq.exp()
        # the rest's share of each token outside the list, given that it is outside
        among = torch.where(inside, -math.inf, logq)
        log_rest = torch.logsumexp(among, 1, keepdim=True)
        target = target + rest * (among - log_rest).exp()
        losses.append(-(torch.where(inside, target * logq, 0.0).sum(1) + (rest * log_rest)[:, 0]))
        grad[sr] = ((q * target.sum(1, keepdim=True) - target) / (N * T)).float()
    pair_loss = torch.cat(losses)
    return pair_loss.mean().reshape(1), pair_loss, grad
