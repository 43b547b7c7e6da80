"""The operators around the routed experts of a decoder layer, as cases that can be timed and compared.

A serving step appends its new tokens' keys and values to a paged cache (the rotation by position applied on
the way), attends from them over that cache, runs the experts, and at the end samples a token from the logits.
A case is one call of one of the three: op "append", "attend" or "sample".

Keys of an append / attend case: seqs, new (tokens a sequence adds), ctx (tokens cached before them), ragged
(lengths vary from sequence to sequence, up to the given ones), hq and hkv heads, d head dimension, dtype, page
(tokens a page), heads_first (a page holds [head][token] in place of [token][head]), rot (dimensions that are
rotated), interleaved, axes (position axes), window (0: none), causal.  Of a sample case: rows, vocab, dtype,
cut (rows have temperature, top-k, top-p and min-p of their own; False: temperature alone), banned (share of
the vocabulary that a grammar forbids).
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
CACHE = dict(op="attend", seqs=1, new=1, ctx=0, ragged=False, hq=32, hkv=8, d=128, dtype="bf16", page=16,
             heads_first=False, window=0, causal=True)
ROPE = dict(rot=128, interleaved=False, axes=1)
MAX_POS = 32768  # rows of the rotation's tables


def listed():
    return [
        # the smallest append: one decoded token of one stream, a small model's heads
        dict(CACHE, **ROPE, name="append_1", op="append", ctx=777, hq=16, hkv=2),
        # a chunk of an image prompt: three ragged sequences, three position axes, a quarter of the head rotated
        dict(CACHE, name="append_chunk_axes", op="append", seqs=3, new=2731, ctx=500, ragged=True, hq=16, hkv=4, d=256,
             page=64, rot=64, interleaved=False, axes=3),
        # one decoded token of one stream over a short context: latency
        dict(CACHE, name="decode_1k", ctx=1000),
        # one decoded token of 64 streams of very different lengths
        dict(CACHE, name="decode_64_ragged", seqs=64, ctx=8191, ragged=True, hkv=4, page=32),
        # one decoded token over a very long context, few wide heads
        dict(CACHE, name="decode_131k", ctx=131070, hq=16, hkv=2, d=256, page=64),
        # speculative verification: five tokens a stream, a sliding window
        dict(CACHE, name="verify_5", seqs=16, new=5, ctx=4093, ragged=True, hkv=4, d=64, dtype="f16", page=24, window=1024),
        # a prefill chunk over what was cached before
        dict(CACHE, name="chunk_2048_16k", new=2048, ctx=14336, page=16, heads_first=True),
        # the prompts of eight users at once, odd lengths
        dict(CACHE, name="prefill_ragged", seqs=8, new=4001, ragged=True, hq=32, hkv=4, dtype="f16", page=64),
        # a prompt through a layer of wide heads with a sliding window
        dict(CACHE, name="prefill_window", new=8192, hq=16, hkv=8, d=256, page=32, window=1024),
        # one row of logits, as a single stream's step ends
        dict(name="sample_1", op="sample", rows=1, vocab=131072, dtype="f32", cut=True, banned=0.0),
        # a batch of streams, each with settings of its own, the largest vocabulary
        dict(name="sample_64", op="sample", rows=64, vocab=262144, dtype="bf16", cut=True, banned=0.1),
        # many rows by temperature alone: nothing is cut, every entry competes
        dict(name="sample_256_plain", op="sample", rows=256, vocab=50001, dtype="f16", cut=False, banned=0.0),
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def _plain_size(n):
    return n + 1 if n == 3072 else n


def _cost(c):
    """(scores, cache values) of an attend case."""
    return c["seqs"] * c["hq"] * c["new"] * (c["ctx"] + c["new"]), c["seqs"] * c["hkv"] * c["d"] * (c["ctx"] + c["new"])


def draw(rng):
    while True:
        kind = rng.choice(("append", "decode", "decode", "verify", "chunk", "prefill", "sample", "sample"))
        if kind == "sample":
            rows, vocab = _log(rng, 1, 256), _plain_size(_log(rng, 1000, 262144))
            if rows * vocab > 64 * 262144:
                continue
            return dict(op="sample", rows=rows, vocab=vocab, dtype=rng.choice(("bf16", "f16", "f32")),
                        cut=rng.random() < 0.75, banned=rng.choice((0.0, 0.1, 0.9)))
        hkv, group, d = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 5, 7, 8, 16)), rng.choice((64, 128, 256))
        c = dict(CACHE, hkv=hkv, hq=hkv * group, d=d, dtype=rng.choice(("bf16", "f16")), ragged=rng.random() < 0.6,
                 page=rng.choice((1, 8, 16, 24, 32, 64, 128)), heads_first=rng.random() < 0.3)
        if c["hq"] > 64 or (c["hq"] + 2 * hkv) * d == 3072:
            continue
        if kind == "append":
            c.update(op="append", seqs=_log(rng, 1, 64), new=rng.choice((1, _plain_size(_log(rng, 1, 4096)))),
                     ctx=_log(rng, 1, 1000), rot=rng.choice((d, d // 2, d // 4)), interleaved=rng.random() < 0.4,
                     axes=rng.choice((1, 1, 3)))
            c["page"] = rng.choice((8, 16, 32, 64))
            if c["seqs"] * (c["new"] + c["ctx"]) * c["hq"] * d > 8192 * 16 * 256:
                continue
            return c
        if kind == "decode":
            c.update(seqs=_log(rng, 1, 128), ctx=_log(rng, 1, 131070))
        elif kind == "verify":
            c.update(seqs=_log(rng, 1, 64), new=rng.randint(2, 16), ctx=_log(rng, 16, 16384))
        elif kind == "chunk":
            c.update(seqs=rng.choice((1, 1, 2, 4)), new=_plain_size(_log(rng, 32, 2048)), ctx=_log(rng, 256, 16384))
        else:
            c.update(seqs=_log(rng, 1, 8), new=_plain_size(_log(rng, 64, 8192)), causal=rng.random() < 0.85)
        if c["causal"] and rng.random() < 0.3:
            c["window"] = rng.choice((128, 1000, 1024, 4096))
        scores, values = _cost(c)
        if scores > 32 * 2048 * 16384 or scores * d > 32 * 2048 * 16384 * 128 or values > 64 * 4 * 128 * 8192:
            continue
        if c["hq"] * c["new"] * c["seqs"] * d > 1 << 27 or 3072 in (c["ctx"], c["ctx"] + c["new"]):
            continue
        return c


# ---- inputs

def _lengths(c):
    """(new tokens, tokens cached before) of each sequence: a part of the case, whatever the seed."""
    n, new, ctx = c["seqs"], [c["new"]] * c["seqs"], [c["ctx"]] * c["seqs"]
    if c["ragged"]:
        u = torch.rand(2, n, generator=torch.Generator().manual_seed(n * 31 + c["new"])).tolist()
        new = [max(1, round(x * (0.2 + 0.8 * r))) for x, r in zip(new, u[0])]
        ctx = [round(x * (0.02 + 0.98 * r * r)) for x, r in zip(ctx, u[1])]
        new[0], ctx[-1] = c["new"], c["ctx"]
    return new, ctx


def _cache_inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed * 7919 + 17)
    dt, d, hq, hkv, page = DTYPES[c["dtype"]], c["d"], c["hq"], c["hkv"], c["page"]
    new, ctx = _lengths(c)
    total = [a + b for a, b in zip(new, ctx)]
    need = [-(-t // page) for t in total]
    n_pages = sum(need) + 3  # some of the pool belongs to others
    perm = torch.randperm(n_pages, device="cuda", generator=g).int()
    table = torch.zeros(c["seqs"], max(need), dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = perm[at:at + n]
        at += n
    shape = (n_pages, hkv, page, d) if c["heads_first"] else (n_pages, page, hkv, d)
    caches = []
    for _ in range(2):
        buf = torch.randn(shape, dtype=dt, device="cuda", generator=g)
        buf[perm[at:].long()] = math.nan  # pages that belong to nobody hold anything
        caches.append(buf.transpose(1, 2) if c["heads_first"] else buf)  # [page][line][head][dim]
    i32 = dict(dtype=torch.int32, device="cuda")
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s = dict(c=c, k_cache=caches[0], v_cache=caches[1], table=table, q_start=torch.tensor(starts, **i32),
             kv_len=torch.tensor(total, **i32), tokens=starts[-1], max_q=max(new))
    T = starts[-1]
    # q, k and v as the fused projection leaves them: one row a token
    qkv = torch.randn(T, (hq + 2 * hkv) * d, dtype=dt, device="cuda", generator=g)
    s["q"] = qkv[:, :hq * d].unflatten(1, (hq, d))
    if c["op"] == "append":
        s["k"] = qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
        s["v"] = qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d))
        half = c["rot"] // 2
        f = 1e4 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        ang = torch.arange(MAX_POS, device="cuda", dtype=torch.float64)[:, None] * f
        s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
        s["pos"] = None
        if c["axes"] > 1:
            s["axis"] = torch.repeat_interleave(torch.arange(c["axes"]), torch.tensor(_sections(c))).cuda()
            s["pos"] = torch.randint(0, MAX_POS, (c["axes"], T), device="cuda", generator=g, dtype=torch.int32)
        s["q_out"] = torch.empty(T, hq, d, dtype=dt, device="cuda")
    else:
        s["q"].mul_(1.5)
        s["scale"] = 1 / math.sqrt(d)
        # each sequence's newest line ends inside a page, what follows in it was never written
        line = torch.arange(max(need) * page, device="cuda")
        for cache in caches:
            for i, t in enumerate(total):
                if t % page:
                    cache[table[i, need[i] - 1].long(), t % page:] = math.nan
        del line
        s["out"] = torch.empty(T, hq, d, dtype=dt, device="cuda")
        s["lse"] = torch.empty(T, hq, device="cuda")
    return s


def _sample_inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed * 7919 + 17)
    n, v = c["rows"], c["vocab"]
    x = torch.randn(n, v, device="cuda", generator=g) * 2.5
    heads = torch.randint(0, v, (n, 32), device="cuda", generator=g)  # the few words that fit
    x.scatter_(1, heads, 8 + 4 * torch.randn(n, 32, device="cuda", generator=g))
    if c["banned"]:
        x.masked_fill_(torch.rand(n, v, device="cuda", generator=g) < c["banned"], -math.inf)
    u = torch.rand(n, v, device="cuda", generator=g).clamp_(1e-10, 1 - 1e-7)
    s = dict(c=c, logits=x.to(DTYPES[c["dtype"]]), noise=-torch.log(-torch.log(u)))

    def pick(*values):
        return torch.tensor(values, device="cuda")[torch.randint(0, len(values), (n,), device="cuda", generator=g)]

    s["temperature"] = pick(0.6, 0.8, 1.0, 1.3)
    s["top_k"] = s["top_p"] = s["min_p"] = None
    if c["cut"]:
        s["temperature"] = pick(0.0, 0.6, 0.7, 0.8, 1.0, 1.0, 1.3) if n > 1 else s["temperature"]
        s["top_k"] = pick(0, 20, 50, 50, 1000).int()
        s["top_p"] = pick(0.8, 0.9, 0.95, 0.99, 1.0)
        s["min_p"] = pick(0.0, 0.0, 0.02, 0.1)
    s["token"] = torch.empty(n, dtype=torch.int32, device="cuda")
    s["logprob"] = torch.empty(n, device="cuda")
    return s


def _inputs(c, seed):
    return _sample_inputs(c, seed) if c["op"] == "sample" else _cache_inputs(c, seed)


class _Handle:
    """The attention workspace that a program keeps."""

    def __init__(self, mf, c, tokens):
        self.mf = mf
        self.at = mf.mf_attn_create(mf.AttnShape(c["hq"], c["hkv"], c["d"], mf.MF_BF16 if c["dtype"] == "bf16" else mf.MF_F16),
                                    c["seqs"], tokens, torch.cuda.current_device())

    def __del__(self):
        self.mf.mf_attn_destroy(self.at)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the handle and the descriptions of its buffers that a serving program holds over its steps
        import paper_2607_09686_gb300 as mf
        s["mf"] = mf
        if case["op"] != "sample":
            s["handle"] = _Handle(mf, case, s["tokens"])
            s["cache"] = mf.kv_cache(s["k_cache"], s["v_cache"])
            s["step"] = mf.step(s["q_start"], s["kv_len"], s["table"], s["tokens"], s["max_q"])
        if case["op"] == "append":
            s["rope"] = mf.rope(s["cos"], s["sin"], s["pos"], interleaved=case["interleaved"],
                                sections=_sections(case))
    return s


# ---- one pass

def run(s):
    op = s["c"]["op"]
    if own:
        mf = s["mf"]
        if op == "append":
            mf.mf_kv_append(s["handle"].at, s["cache"], s["step"], s["k"], s["v"], s["q"], s["q_out"], s["rope"])
            return s["q_out"], s["k_cache"], s["v_cache"]
        if op == "attend":
            mf.mf_attn_forward(s["handle"].at, s["cache"], s["step"], s["q"], s["out"], s["lse"], s["scale"],
                               window=s["c"]["window"], causal=s["c"]["causal"])
            return s["out"], s["lse"]
        mf.mf_sample(s["logits"], s["noise"], s["token"], s["logprob"], s["temperature"], s["top_k"], s["top_p"],
                     s["min_p"])
        return s["token"], s["logprob"]
    return {"append": _append, "attend": _attend, "sample": _sample}[op](s)


def _sections(c):
    """Pairs of each axis: a quarter for the time, the rest for height and width."""
    half = c["rot"] // 2
    if c["axes"] == 1:
        return (half,)
    side = (half - half // 4) // 2
    return (half - 2 * side, side, side)


def _tokens(s):
    """Per new token: its sequence and its position in the cache."""
    t = torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(s["q_start"], t, right=True) - 1
    new = s["q_start"][1:] - s["q_start"][:-1]
    return seq, (s["kv_len"] - new)[seq] + t - s["q_start"][seq]


def _rotate(x, cos, sin, rot, interleaved):
    """x [T][heads][d] in 32 bits, cos and sin [T][rot / 2]."""
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., ::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    cos, sin = cos[:, None], sin[:, None]
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((r, rest), -1)


def _append(s):
    c = s["c"]
    seq, at = _tokens(s)
    if s["pos"] is None:
        cos, sin = s["cos"][at], s["sin"][at]
    else:  # pair j turns by the position on its section's axis
        p = s["pos"][s["axis"]].t().long()  # [T][pairs]
        pair = torch.arange(c["rot"] // 2, device="cuda")
        cos, sin = s["cos"][p, pair], s["sin"][p, pair]
    dt = s["q"].dtype
    q = _rotate(s["q"].float(), cos, sin, c["rot"], c["interleaved"]).to(dt)
    k = _rotate(s["k"].float(), cos, sin, c["rot"], c["interleaved"]).to(dt)
    page = s["table"][seq, at // c["page"]].long()
    s["k_cache"][page, at % c["page"]] = k
    s["v_cache"][page, at % c["page"]] = s["v"]
    return q, s["k_cache"], s["v_cache"]


def _attend(s):
    c, page = s["c"], s["c"]["page"]
    n, hkv, group, d = c["seqs"], c["hkv"], c["hq"] // c["hkv"], c["d"]
    longest, most = s["table"].shape[1] * page, s["max_q"]
    line = torch.arange(longest, device="cuda")
    held = line < s["kv_len"][:, None]  # [n][longest]
    at = s["table"].long()[:, line // page]
    k, v = (torch.where(held[:, :, None, None], x[at, line % page], 0).float() for x in (s["k_cache"], s["v_cache"]))
    seq, pos = _tokens(s)
    t = torch.arange(s["tokens"], device="cuda") - s["q_start"][seq]
    q = torch.zeros(n, most, hkv, group, d, device="cuda")
    q[seq, t] = s["q"].float().unflatten(1, (hkv, group))
    see = torch.zeros(n, most, longest, dtype=torch.bool, device="cuda")
    see[seq, t] = (line <= pos[:, None] if c["causal"] else held[seq]) & (line > pos[:, None] - (c["window"] or longest + 1))
    x = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(n, hkv, group * most, d), k.permute(0, 2, 3, 1)).mul_(s["scale"])
    x = x.view(n, hkv, group, most, longest).masked_fill_(~see[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(m == -math.inf, 0, m)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(n, hkv, group * most, longest), v.transpose(1, 2)).view(n, hkv, group, most, d)
    out = out / torch.where(total == 0, 1, total)
    lse = (m + total.log()).squeeze(-1)
    out, lse = out.permute(0, 3, 1, 2, 4)[seq, t], lse.permute(0, 3, 1, 2)[seq, t]
    return out.flatten(1, 2).to(s["q"].dtype), lse.flatten(1, 2).contiguous()


def _sample(s):
    x = s["logits"].float()
    n, v = x.shape
    x = torch.where(x.isnan(), -math.inf, x)
    m = x.amax(-1, keepdim=True)
    t = s["temperature"][:, None]
    greedy = ~(t > 0)
    x, order = x.sort(dim=-1, descending=True, stable=True)
    z = torch.where(x == m, 0, (x - m) / torch.where(greedy, 1, t))
    w = z.exp()
    rank = torch.arange(v, device="cuda")
    keep = (x > -math.inf) & (~greedy | (rank == 0))
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        keep &= (k <= 0) | (rank < k)
    if s["top_p"] is not None:
        p = s["top_p"][:, None]
        mass = w * keep
        keep &= (mass.cumsum(-1) - mass < p * mass.sum(-1, keepdim=True)) | (p >= 1) | (rank == 0)
    if s["min_p"] is not None:
        keep &= (w >= s["min_p"][:, None]) | (rank == 0)
    g = s["noise"].gather(1, order)
    key = torch.where(keep, z + torch.where(g.isnan(), -math.inf, g), -math.inf)
    token = torch.where(keep & (key == key.amax(-1, keepdim=True)), order, v).amin(-1, keepdim=True)
    chosen = torch.where(order == token, z, 0).sum(-1)
    logprob = chosen - (w * keep).sum(-1).log()
    none = token[:, 0] == v
    return torch.where(none, -1, token[:, 0]).int(), torch.where(none, -math.inf, logprob)


# ---- the definitions, in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    return {"append": _append64, "attend": _attend64, "sample": _sample64}[case["op"]](s)


def _rows64(s):
    """Per sequence: the slice of its new tokens, its length in the cache, and the (page, line) of each position."""
    start, total, table, page = s["q_start"].tolist(), s["kv_len"].tolist(), s["table"].long(), s["c"]["page"]
    for i, n in enumerate(total):
        at = torch.arange(n, device="cuda")
        yield slice(start[i], start[i + 1]), n, table[i, at // page], at % page


def _append64(s):
    c = s["c"]
    rot, half = c["rot"], c["rot"] // 2
    bounds = [0]
    for n in _sections(c):
        bounds.append(bounds[-1] + n)
    q, k = s["q"].double(), s["k"].double()
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    for new, n, page, line in _rows64(s):
        fresh = new.stop - new.start
        at = torch.arange(n - fresh, n, device="cuda")
        for x in (q, k):
            for a in range(len(bounds) - 1):
                p = at if s["pos"] is None else s["pos"][a, new].long()
                for j in range(bounds[a], bounds[a + 1]):
                    i0, i1 = (2 * j, 2 * j + 1) if c["interleaved"] else (j, j + half)
                    turn = torch.complex(s["cos"][p, j].double(), s["sin"][p, j].double())[:, None]
                    y = torch.complex(x[new, :, i0], x[new, :, i1]) * turn
                    x[new, :, i0], x[new, :, i1] = y.real, y.imag
        kc[page[n - fresh:], line[n - fresh:]] = k[new]
        vc[page[n - fresh:], line[n - fresh:]] = s["v"][new].double()
    return q, kc, vc


def _attend64(s):
    c = s["c"]
    if _cost(c)[0] * c["d"] * 4 > 6e12:
        return None
    group = c["hq"] // c["hkv"]
    out = torch.zeros(s["tokens"], c["hq"], c["d"], dtype=torch.float64, device="cuda")
    lse = torch.full((s["tokens"], c["hq"]), -math.inf, dtype=torch.float64, device="cuda")
    for new, n, page, line in _rows64(s):
        at = torch.arange(n, device="cuda")
        pos = at[n - (new.stop - new.start):, None]
        hidden = torch.zeros(len(pos), n, dtype=torch.bool, device="cuda")
        if c["causal"]:
            hidden |= at > pos
        if c["window"]:
            hidden |= at <= pos - c["window"]
        for h in range(c["hkv"]):
            k, v = s["k_cache"][page, line, h].double(), s["v_cache"][page, line, h].double()
            for g in range(h * group, (h + 1) * group):
                x = s["scale"] * (s["q"][new, g].double() @ k.t())
                x[hidden] = -math.inf
                lse[new, g] = torch.logsumexp(x, -1)
                out[new, g] = torch.exp(x - lse[new, g, None]) @ v
    return out, lse


def _sample64(s):
    x = s["logits"].double().nan_to_num(-math.inf, math.inf, -math.inf)
    t, g = s["temperature"].double().tolist(), s["noise"].double()
    result = []
    for i, row in enumerate(x):
        best = row.max()
        if t[i] > 0:
            z = torch.where(row == best, 0, (row - best) / t[i])
        else:
            z = torch.where(torch.arange(len(row), device="cuda") == row.argmax(), 0.0, -math.inf).double()
        order = torch.argsort(z, dim=-1, descending=True, stable=True)
        w = z[order].exp()
        n = int((z[order] > -math.inf).sum())
        if s["top_k"] is not None and s["top_k"][i] > 0:
            n = min(n, int(s["top_k"][i]))
        if s["top_p"] is not None and s["top_p"][i] < 1:
            n_p = int((w[:n].cumsum(0) < float(s["top_p"][i]) * w[:n].sum()).sum()) + 1
        else:
            n_p = n
        if s["min_p"] is not None:
            n = min(n, int((w >= float(s["min_p"][i])).sum()))
        kept = order[:max(1, min(n, n_p))]
        token = kept[(z[kept] + g[i, kept]).argmax()]
        result.append(z[token] - z[kept].exp().sum().log())
    return None, torch.stack(result)


# ---- the work that a call cannot do without

def work(c):
    if c["op"] == "sample":
        e = 4 if c["dtype"] == "f32" else 2
        n = c["rows"] * c["vocab"]
        return {"bytes": n * e + (0 if c["cut"] else n * 4) + 28 * c["rows"], "flops": n * 4}
    new, ctx = _lengths(c)
    tokens, e, d = sum(new), 2, c["d"]
    if c["op"] == "append":
        return {"bytes": tokens * (2 * (c["hq"] + 2 * c["hkv"]) * d * e + c["rot"] * 4 + 8), "flops": tokens * (c["hq"] + c["hkv"]) * c["rot"] * 3}
    keys = pairs = 0
    for n, before in zip(new, ctx):
        w = c["window"] or before + n
        keys += min(before + n, n + w)
        if c["causal"]:  # token i sees min(before + i + 1, w) keys
            full = max(0, min(n, w - before))  # tokens whose window is not yet full
            pairs += full * before + full * (full + 1) // 2 + (n - full) * w
        else:
            pairs += n * (before + n)
    return {"bytes": 2 * tokens * c["hq"] * d * e + tokens * c["hq"] * 4 + 2 * keys * c["hkv"] * d * e, "flops": 4 * pairs * c["hq"] * d}
