"""Operators of a serving step whose streams share a prompt and are drafted ahead, as cases that can be timed and compared.

Three operators: the append to a paged cache with the norms of queries and keys (each head's root mean square) and the rotation in
the same pass; attention of a batch whose groups of streams share their first lines, which are read once for the group; and the
verification of drafted tokens against the target's probabilities, with random numbers given.  A case is one call of one of them: op
"norm", "shared" or "verify".

Keys of a norm case: seqs, new (tokens a sequence adds), ctx (tokens cached before them), ragged (lengths vary, up to the given
ones), hq and hkv heads, d head dimension, dtype, page (tokens a page), heads_first (a page holds [head][token] in place of
[token][head]), rot (dimensions that are rotated), interleaved, axes (position axes), offset (added to the weights).  Of a shared case,
besides: groups, seqs (of a group), prefix (tokens that a group shares), ctx (tokens of a sequence's own before the new ones).  Of a verify
case: seqs, drafts (the most a sequence has), ragged, vocab, dtype, model (the drafter gives logits; False: the drafts are
certain, as looked up in what was said before), cut (top-k, top-p and min-p; False: temperature alone).
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
CACHE = dict(seqs=1, new=1, ctx=0, ragged=False, hq=32, hkv=4, d=128, dtype="bf16", page=16, heads_first=False)
NORM = dict(CACHE, op="norm", rot=128, interleaved=False, axes=1, offset=0.0)
SHARED = dict(CACHE, op="shared", groups=1, prefix=0)
VERIFY = dict(op="verify", seqs=1, drafts=4, ragged=False, vocab=131072, dtype="bf16", model=True, cut=False)
MAX_POS = 32768  # rows of the rotation's tables
EPS = 1e-6


def listed():
    return [
        # one decoded token of one stream, a small model's heads: latency
        dict(NORM, name="norm_1", ctx=777, hq=16, hkv=2),
        # single tokens of 64 streams, head weights that are kept less one
        dict(NORM, name="norm_64", seqs=64, ctx=900, ragged=True, page=32, offset=1.0),
        # an image prompt's chunk: three ragged sequences, three position axes, a quarter of the head rotated
        dict(NORM, name="norm_chunk_axes", seqs=3, new=2731, ctx=500, ragged=True, hq=16, hkv=4, d=256, page=64, rot=64, axes=3,
             dtype="f16", interleaved=True, heads_first=True),
        # a prefill chunk
        dict(NORM, name="norm_chunk", new=8192, ctx=1000, page=64),
        # two streams after a system prompt of a page or so: latency
        dict(SHARED, name="shared_2_1k", seqs=2, ctx=37, prefix=1000, ragged=True),
        # 64 streams, one token each, after a long document that all of them ask about
        dict(SHARED, name="shared_64_16k", seqs=64, ctx=1000, prefix=16384, ragged=True),
        # verification batches in four groups with a prompt each, small heads
        dict(SHARED, name="shared_verify", groups=4, seqs=12, new=5, ctx=500, prefix=4093, ragged=True, hq=32, hkv=8, d=64, dtype="f16",
             page=24),
        # the questions of eight users about one document, wide heads
        dict(SHARED, name="shared_prompts", seqs=8, new=701, prefix=8192, ragged=True, hq=16, hkv=2, d=256, page=64, heads_first=True),
        # one stream, four drafted tokens: latency
        dict(VERIFY, name="verify_1", dtype="f32", cut=True),
        # a batch of streams by temperature alone
        dict(VERIFY, name="verify_64", seqs=64, ragged=True),
        # streams with settings of their own, a large vocabulary
        dict(VERIFY, name="verify_cut", seqs=24, ragged=True, vocab=200001, dtype="f16", cut=True),
        # drafts looked up in the text, more of them, certain
        dict(VERIFY, name="verify_lookup", seqs=64, drafts=8, ragged=True, vocab=50001, model=False),
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def _scores(c):
    """Products of a query with a key, of the longest sequences."""
    return c["groups"] * c["seqs"] * c["new"] * c["hq"] * (c["prefix"] + c["ctx"] + c["new"])


def draw(rng):
    while True:
        op = rng.choice(("norm", "shared", "shared", "verify"))
        if op == "verify":
            c = dict(VERIFY, seqs=_log(rng, 1, 64), drafts=rng.randint(1, 8), ragged=rng.random() < 0.7, vocab=_log(rng, 1000, 262144),
                     dtype=rng.choice(("bf16", "f16", "f32")), model=rng.random() < 0.6, cut=rng.random() < 0.5)
            if c["seqs"] * (c["drafts"] + 1) * c["vocab"] > (24 if c["cut"] else 64) * 5 * 131072:
                continue
            return c
        hkv, group, d = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 5, 8, 16)), rng.choice((64, 128, 256))
        heads = dict(hkv=hkv, hq=hkv * group, d=d, dtype=rng.choice(("bf16", "f16")), page=rng.choice((8, 16, 24, 32, 64, 128)),
                     heads_first=rng.random() < 0.3)
        if hkv * group > 64:
            continue
        if op == "norm":
            c = dict(NORM, seqs=_log(rng, 1, 64), new=rng.choice((1, _log(rng, 1, 8192))), ctx=_log(rng, 1, 1000),
                     ragged=rng.random() < 0.6, interleaved=rng.random() < 0.4, axes=rng.choice((1, 1, 3)), offset=rng.choice((0.0, 1.0)))
            c.update(heads, rot=rng.choice((d, d // 2, d // 4)))
            if c["seqs"] * (c["new"] + c["ctx"]) * c["hq"] * d > 9192 * 32 * 128:
                continue
            return c
        kind = rng.choice(("decode", "decode", "verify", "prompts"))
        c = dict(SHARED, groups=rng.choice((1, 1, 2, 4)), ragged=rng.random() < 0.7)
        c.update(heads)
        if kind == "prompts":
            c.update(seqs=_log(rng, 2, 8), new=_log(rng, 32, 1000), prefix=_log(rng, 256, 8192), ctx=rng.choice((0, 0, 100)))
        else:
            c.update(seqs=_log(rng, 2, 64), new=1 if kind == "decode" else rng.randint(2, 8), prefix=_log(rng, 64, 32768),
                     ctx=_log(rng, 1, 1000))
        lines = c["groups"] * (c["prefix"] + c["seqs"] * (c["ctx"] + c["new"])) * hkv * d
        if _scores(c) * d > 8 * 701 * 16 * 8893 * 256 or lines > (16384 + 64 * 1001) * 4 * 128:
            continue
        return c


# ---- inputs

def _lengths(c):
    """(new tokens, own tokens cached before) of each sequence: a part of the case, whatever the seed."""
    n = c["seqs"] * c.get("groups", 1)
    new, ctx = [c["new"]] * n, [c["ctx"]] * n
    if c["ragged"]:
        u = torch.rand(2, n, generator=torch.Generator().manual_seed(n * 31 + c["new"])).tolist()
        new = [max(1, round(x * (0.2 + 0.8 * r))) for x, r in zip(new, u[0])]
        ctx = [round(x * (0.02 + 0.98 * r * r)) for x, r in zip(ctx, u[1])]
        new[0], ctx[-1] = c["new"], c["ctx"]
    return new, ctx


def _cache_inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed * 7919 + 17)
    dt, d, hq, hkv, page = DTYPES[c["dtype"]], c["d"], c["hq"], c["hkv"], c["page"]
    prefix, groups = c.get("prefix", 0), c.get("groups", 1)
    new, own_ctx = _lengths(c)
    total = [prefix + a + b for a, b in zip(new, own_ctx)]
    whole = prefix // page  # pages of a prefix that its sequences hold in common
    need = [-(-t // page) for t in total]
    n_pages = whole * groups + sum(x - whole for x in need) + 3  # some of the pool belongs to others
    perm = torch.randperm(n_pages, device="cuda", generator=g).int()
    table = torch.zeros(len(new), max(need), dtype=torch.int32, device="cuda")
    at = whole * groups
    for i, n in enumerate(need):
        of = i // c["seqs"] * whole
        table[i, :whole] = perm[of:of + whole]
        table[i, whole:n] = perm[at:at + n - whole]
        at += n - whole
    shape = (n_pages, hkv, page, d) if c["heads_first"] else (n_pages, page, hkv, d)
    caches = []
    for _ in range(2):
        buf = torch.randn(shape, dtype=dt, device="cuda", generator=g)
        buf[perm[at:].long()] = math.nan  # pages that belong to nobody hold anything
        caches.append(buf.transpose(1, 2) if c["heads_first"] else buf)  # [page][line][head][dim]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    i32 = dict(dtype=torch.int32, device="cuda")
    T = starts[-1]
    s = dict(c=c, k_cache=caches[0], v_cache=caches[1], table=table, q_start=torch.tensor(starts, **i32),
             kv_len=torch.tensor(total, **i32), tokens=T, max_q=max(new), new=new, total=total)
    # q, k and v as the fused projection leaves them: one row a token
    qkv = torch.randn(T, (hq + 2 * hkv) * d, dtype=dt, device="cuda", generator=g)
    s["q"] = qkv[:, :hq * d].unflatten(1, (hq, d))
    if c["op"] == "norm":
        qkv.mul_(3 * torch.rand(T, 1, device="cuda", generator=g) + 0.1)  # tokens of very different size
        s["k"] = qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
        s["v"] = qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d))
        for name in ("q_weight", "k_weight"):
            s[name] = (1 - c["offset"] + 0.3 * torch.randn(d, device="cuda", generator=g)).to(dt)
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
        for cache in caches:
            for i, t in enumerate(total):
                # what follows a sequence's newest line in its page was never written; what its own pages hold of the prefix is
                # the group's
                if t % page:
                    cache[table[i, need[i] - 1].long(), t % page:] = math.nan
                if prefix % page and i % c["seqs"]:
                    first = i - i % c["seqs"]
                    cache[table[i, whole].long(), :prefix % page] = cache[table[first, whole].long(), :prefix % page]
        s["first"] = torch.arange(groups + 1, **i32) * c["seqs"]
        s["shared"] = torch.full((groups,), prefix, **i32)
        s["out"] = torch.empty(T, hq, d, dtype=dt, device="cuda")
        s["lse"] = torch.empty(T, hq, device="cuda")
    return s


def _gumbel(shape, g):
    u = torch.rand(shape, device="cuda", generator=g).clamp_(1e-10, 1 - 1e-7)
    return u.log_().neg_().log_().neg_()


def _verify_inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed * 7919 + 17)
    n, v = c["seqs"], c["vocab"]
    rows = [c["drafts"] + 1] * n
    if c["ragged"]:
        u = torch.rand(n, generator=torch.Generator().manual_seed(n * 31 + v)).tolist()
        rows = [1 + max(0, round(c["drafts"] * (1.2 * x - 0.1))) for x in u]
        rows = [min(r, c["drafts"] + 1) for r in rows]
        rows[0] = c["drafts"] + 1
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
    R = starts[-1]
    x = torch.randn(R, v, device="cuda", generator=g) * 2.5
    heads = torch.randint(0, v, (R, 32), device="cuda", generator=g)  # the few words that fit
    x.scatter_(1, heads, 8 + 4 * torch.randn(R, 32, device="cuda", generator=g))
    s = dict(c=c, logits=x.to(DTYPES[c["dtype"]]), row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), starts=starts)
    x += 0.7 * torch.randn(R, v, device="cuda", generator=g)  # the drafter is of much the same opinion
    s["draft_logits"] = x.to(DTYPES[c["dtype"]]) if c["model"] else None

    def pick(*values):
        return torch.tensor(values, device="cuda")[torch.randint(0, len(values), (n,), device="cuda", generator=g)]

    s["cuts"] = dict(temperature=pick(0.6, 0.8, 1.0, 1.3), top_k=None, top_p=None, min_p=None)
    if c["cut"]:
        s["cuts"] = dict(temperature=pick(0.0, 0.6, 0.7, 0.8, 1.0, 1.0, 1.3) if n > 1 else pick(0.7, 0.8, 1.0),
                         top_k=pick(0, 20, 50, 50, 1000).int(), top_p=pick(0.8, 0.9, 0.95, 0.99, 1.0), min_p=pick(0.0, 0.0, 0.02, 0.1))
    # the drafter's tokens: drawn from its own logits with the stream's settings, or likely ones
    s["draft_cuts"] = s["cuts"]
    seq = torch.searchsorted(s["row_start"], torch.arange(R, device="cuda"), right=True) - 1
    if c["model"]:
        p, _ = _probabilities(s["draft_logits"], s["cuts"], seq)
        drawn = (p.log() + _gumbel((R, v), g)).argmax(-1)
    else:
        drawn = torch.where(torch.rand(R, device="cuda", generator=g) < 0.7, x.argmax(-1), torch.randint(0, v, (R,), device="cuda", generator=g))
    s["tokens"] = torch.cat((torch.zeros(1, device="cuda"), drawn[:-1])).int()  # the step's input: row i's draft is token i + 1
    s["u"] = torch.rand(R, device="cuda", generator=g)
    s["noise"] = _gumbel((n, v), g)
    s["token"] = torch.empty(R, dtype=torch.int32, device="cuda")
    s["accepted"] = torch.empty(n, dtype=torch.int32, device="cuda")
    s["logprob"] = torch.empty(R, device="cuda")
    return s


def _inputs(c, seed):
    return _verify_inputs(c, seed) if c["op"] == "verify" else _cache_inputs(c, seed)


class _Handle:
    """The attention workspace that a program keeps."""

    def __init__(self, mf, c, seqs, tokens):
        self.mf = mf
        self.at = mf.mf_attn_create(mf.AttnShape(c["hq"], c["hkv"], c["d"], mf.MF_BF16 if c["dtype"] == "bf16" else mf.MF_F16),
                                    seqs, tokens, torch.cuda.current_device())

    def __del__(self):
        self.mf.mf_attn_destroy(self.at)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the handle, the workspace and the descriptions of its buffers that a serving program holds over its steps
        import paper_2607_09686_gb300 as mf
        s["mf"] = mf
        if case["op"] == "verify":
            s["cuts"], s["draft_cuts"] = mf.cuts(**s["cuts"]), mf.cuts(**s["draft_cuts"])
            s["work"] = torch.empty(mf.mf_verify_bytes(case["seqs"], s["starts"][-1], case["vocab"]), dtype=torch.uint8, device="cuda")
            return s
        s["handle"] = _Handle(mf, case, len(s["new"]), s["tokens"])
        s["cache"] = mf.kv_cache(s["k_cache"], s["v_cache"])
        s["step"] = mf.step(s["q_start"], s["kv_len"], s["table"], s["tokens"], s["max_q"])
        if case["op"] == "norm":
            s["rope"] = mf.rope(s["cos"], s["sin"], s["pos"], interleaved=case["interleaved"], sections=_sections(case))
            s["norm"] = mf.qk_norm(s["q_weight"], s["k_weight"], EPS, case["offset"])
        else:
            mf.mf_attn_share(s["handle"].at, case["groups"])
            s["groups"] = mf.shared(s["first"], s["shared"])
    return s


# ---- one pass

def run(s):
    op = s["c"]["op"]
    if own:
        mf = s["mf"]
        if op == "norm":
            mf.mf_kv_append_norm(s["handle"].at, s["cache"], s["step"], s["norm"], s["k"], s["v"], s["q"], s["q_out"], s["rope"])
            return s["q_out"], s["k_cache"], s["v_cache"]
        if op == "shared":
            mf.mf_attn_forward_shared(s["handle"].at, s["cache"], s["step"], s["groups"], s["q"], s["out"], s["lse"], s["scale"])
            return s["out"], s["lse"]
        mf.mf_verify(s["logits"], s["row_start"], s["tokens"], s["u"], s["noise"], s["token"], s["accepted"], s["work"], s["logprob"],
                     s["cuts"], s["draft_logits"], s["draft_cuts"])
        return s["token"], s["accepted"], s["logprob"]
    return {"norm": _norm, "shared": _shared, "verify": _verify}[op](s)


def _sections(c):
    """Pairs of each axis: a quarter for the time, the rest for height and width."""
    half = c["rot"] // 2
    if c["axes"] == 1:
        return (half,)
    side = (half - half // 4) // 2
    return (half - 2 * side, side, side)


def _normed(x, weight, offset):
    x = x.float()
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * (weight.float() + offset)


def _rotate(x, cos, sin, rot, interleaved):
    """x [T][heads][d] in 32 bits, cos and sin [T][rot / 2]."""
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., ::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    cos, sin = cos[:, None], sin[:, None]
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((r, rest), -1)


def _norm(s):
    c, t = s["c"], torch.arange(s["tokens"], device="cuda")
    seq = torch.searchsorted(s["q_start"], t, right=True) - 1
    at = (s["kv_len"] - s["q_start"][1:])[seq] + t  # each new token's line in its sequence
    if s["pos"] is None:
        cos, sin = s["cos"][at], s["sin"][at]
    else:  # pair j turns by the position on its section's axis
        p = s["pos"][s["axis"]].t().long()  # [T][pairs]
        pair = torch.arange(c["rot"] // 2, device="cuda")
        cos, sin = s["cos"][p, pair], s["sin"][p, pair]
    dt = s["q"].dtype
    q = _rotate(_normed(s["q"], s["q_weight"], c["offset"]), cos, sin, c["rot"], c["interleaved"]).to(dt)
    k = _rotate(_normed(s["k"], s["k_weight"], c["offset"]), cos, sin, c["rot"], c["interleaved"]).to(dt)
    page = s["table"][seq, at // c["page"]].long()
    s["k_cache"][page, at % c["page"]] = k
    s["v_cache"][page, at % c["page"]] = s["v"]
    return q, s["k_cache"], s["v_cache"]


def _shared(s):
    c, page, group = s["c"], s["c"]["page"], s["c"]["hq"] // s["c"]["hkv"]
    at, outs, sums = 0, [], []
    for i, (n, length) in enumerate(zip(s["new"], s["total"])):
        line = torch.arange(length, device="cuda")
        where = s["table"][i].long()[line // page]
        k, v = (x[where, line % page].float() for x in (s["k_cache"], s["v_cache"]))  # [length][hkv][d]
        q = s["q"][at:at + n].float().unflatten(1, (c["hkv"], group))
        x = torch.matmul(q.permute(1, 2, 0, 3).flatten(1, 2), k.permute(1, 2, 0)).mul_(s["scale"]).unflatten(1, (group, n))
        if n > 1:
            x.masked_fill_(line > line[length - n:, None], -math.inf)
        m = x.amax(-1, keepdim=True)
        p = x.sub_(m).exp_()
        total = p.sum(-1, keepdim=True)
        out = torch.matmul(p.flatten(1, 2), v.transpose(0, 1)).unflatten(1, (group, n)) / total
        outs.append(out.permute(2, 0, 1, 3).flatten(1, 2))
        sums.append((m + total.log()).squeeze(-1).permute(2, 0, 1).flatten(1))
        at += n
    return torch.cat(outs).to(s["q"].dtype), torch.cat(sums)


def _probabilities(logits, cuts, seq):
    """The probabilities of the rows' kept entries and their logarithms, the settings those of row i's sequence seq[i]."""
    x = logits.float()
    n, v = x.shape
    x = torch.where(x.isnan(), -math.inf, x)
    m = x.amax(-1, keepdim=True)
    t = cuts["temperature"][seq][:, None]
    greedy = ~(t > 0)
    z = torch.where(x == m, 0, (x - m) / torch.where(greedy, 1, t))
    keep = x > -math.inf
    if cuts["top_k"] is not None or cuts["top_p"] is not None or cuts["min_p"] is not None:
        z, order = z.sort(dim=-1, descending=True, stable=True)
        w = z.exp()
        rank = torch.arange(v, device="cuda")
        keep = (z > -math.inf) & (~greedy | (rank == 0))
        k, p = cuts["top_k"][seq][:, None], cuts["top_p"][seq][:, None]
        keep &= (k <= 0) | (rank < k)
        mass = w.double() * keep  # (sums beside a border)
        keep &= (mass.cumsum(-1) - mass < p * mass.sum(-1, keepdim=True)) | (p >= 1) | (rank == 0)
        keep &= (w >= cuts["min_p"][seq][:, None]) | (rank == 0)
        total = (w * keep).sum(-1, keepdim=True)
        log_p = torch.empty_like(z).scatter_(1, order, torch.where(keep, z - total.log(), -math.inf))
    else:
        first = torch.arange(v, device="cuda") == x.argmax(-1, keepdim=True)
        z = torch.where(keep & (~greedy | first), z, -math.inf)
        log_p = z - z.exp().sum(-1, keepdim=True).log()
    return log_p.exp(), log_p


def _verify(s):
    n, R = s["c"]["seqs"], len(s["logits"])
    rows, start = torch.arange(R, device="cuda"), s["row_start"].long()
    seq = torch.searchsorted(start, rows, right=True) - 1
    p, log_p = _probabilities(s["logits"], s["cuts"], seq)
    drafted = rows + 1 < start[1:][seq]
    draft = torch.cat((s["tokens"][1:], s["tokens"][:1])).long()
    if s["draft_logits"] is None:
        q = torch.zeros_like(p).scatter_(1, draft[:, None], 1.0)
    else:
        q, _ = _probabilities(s["draft_logits"], s["draft_cuts"], seq)
    at = draft[:, None]
    good = drafted & (s["u"] * q.gather(1, at)[:, 0] < p.gather(1, at)[:, 0])
    # the row after the drafts that were taken, one after the other
    stop = torch.where(good, R, rows)
    last = torch.full((n,), R, device="cuda").scatter_reduce_(0, seq, stop, "amin")
    left = torch.where(drafted[last][:, None], p[last] - q[last], p[last]).clamp_(min=0)
    left = torch.where((left > 0).any(-1, keepdim=True), left, p[last])
    key = torch.where(left > 0, left.log() + s["noise"], -math.inf)
    token = torch.where((left > 0) & (key == key.amax(-1, keepdim=True)), torch.arange(s["c"]["vocab"], device="cuda"), s["c"]["vocab"]).amin(-1)
    out = torch.where(rows < last[seq], draft, -1)
    out[last] = torch.where(token < s["c"]["vocab"], token, -1)
    logprob = torch.where(out >= 0, log_p.gather(1, out.clamp(min=0)[:, None])[:, 0], -math.inf)
    return out.int(), (last - start[:-1]).int(), logprob


# ---- the definitions, in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _norm64, "shared": _shared64, "verify": _verify64}[case["op"]](s)


def _norm64(s):
    c = s["c"]
    rot, half = c["rot"], c["rot"] // 2
    bounds = [0]
    for n in _sections(c):
        bounds.append(bounds[-1] + n)
    q, k = s["q"].double(), s["k"].double()
    for x, w in ((q, s["q_weight"]), (k, s["k_weight"])):
        x /= torch.sqrt((x * x).sum(-1, keepdim=True) / c["d"] + EPS)
        x *= w.double() + c["offset"]
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    begin = 0
    for i, (fresh, n) in enumerate(zip(s["new"], s["total"])):
        new = slice(begin, begin + fresh)
        begin += fresh
        at = torch.arange(n - fresh, n, device="cuda")
        for x in (q, k):
            for a in range(len(bounds) - 1):
                p = at if s["pos"] is None else s["pos"][a, new].long()
                for j in range(bounds[a], bounds[a + 1]):
                    i0, i1 = (2 * j, 2 * j + 1) if c["interleaved"] else (j, j + half)
                    turn = torch.complex(s["cos"][p, j].double(), s["sin"][p, j].double())[:, None]
                    y = torch.complex(x[new, :, i0], x[new, :, i1]) * turn
                    x[new, :, i0], x[new, :, i1] = y.real, y.imag
        page = s["table"][i].long()[at // c["page"]]
        kc[page, at % c["page"]] = k[new]
        vc[page, at % c["page"]] = s["v"][new].double()
    return q, kc, vc


def _shared64(s):
    c = s["c"]
    if _scores(c) * c["d"] * 4 > 3e12:
        return None
    group = c["hq"] // c["hkv"]
    out = torch.zeros(s["tokens"], c["hq"], c["d"], dtype=torch.float64, device="cuda")
    lse = torch.full((s["tokens"], c["hq"]), -math.inf, dtype=torch.float64, device="cuda")
    begin = 0
    for i, (fresh, n) in enumerate(zip(s["new"], s["total"])):
        at = torch.arange(n, device="cuda")
        page, line = s["table"][i].long()[at // c["page"]], at % c["page"]
        new = slice(begin, begin + fresh)
        begin += fresh
        hidden = at > at[n - fresh:, None]
        for h in range(c["hkv"]):
            k, v = s["k_cache"][page, line, h].double(), s["v_cache"][page, line, h].double()
            for g in range(h * group, (h + 1) * group):
                x = s["scale"] * (s["q"][new, g].double() @ k.t())
                x[hidden] = -math.inf
                lse[new, g] = torch.logsumexp(x, -1)
                out[new, g] = torch.exp(x - lse[new, g, None]) @ v
    return out, lse


def _row64(row, cuts, i):
    """log p of one row in 64 bits, settings of sequence i."""
    x = row.double().nan_to_num(-math.inf, math.inf, -math.inf)
    t = float(cuts["temperature"][i])
    order = torch.argsort(x, descending=True, stable=True)
    if not t > 0:
        kept, z = order[:1], x[order[:1]] * 0
    else:
        z = (x[order] - x[order[0]]) / t
        w = z.exp()
        n = int((w > 0).sum())
        if cuts["top_k"] is not None and cuts["top_k"][i] > 0:
            n = min(n, int(cuts["top_k"][i]))
        if cuts["top_p"] is not None and cuts["top_p"][i] < 1:
            n = min(n, int((w[:n].cumsum(0) < float(cuts["top_p"][i]) * w[:n].sum()).sum()) + 1)
        if cuts["min_p"] is not None:
            n = min(n, int((w >= float(cuts["min_p"][i])).sum()))
        kept, z = order[:n], z[:n]
    return torch.full_like(x, -math.inf).scatter_(0, kept, z - z.exp().sum().log())


def _verify64(s):
    tokens, u, starts = s["tokens"].tolist(), s["u"].double().tolist(), s["starts"]
    logprob = torch.full((starts[-1],), -math.inf, dtype=torch.float64, device="cuda")
    for i in range(s["c"]["seqs"]):
        for r in range(starts[i], starts[i + 1]):
            log_p = _row64(s["logits"][r], s["cuts"], i)
            p = log_p.exp()
            rest = p
            if r + 1 < starts[i + 1]:
                x = tokens[r + 1]
                if s["draft_logits"] is None:
                    q = torch.zeros_like(p)
                    q[x] = 1
                else:
                    q = _row64(s["draft_logits"][r], s["draft_cuts"], i).exp()
                if u[r] * float(q[x]) < float(p[x]):
                    logprob[r] = log_p[x]
                    continue
                rest = (p - q).clamp(min=0)
                if not bool((rest > 0).any()):
                    rest = p
            logprob[r] = log_p[(rest.log() + s["noise"][i]).argmax()]
            break
    return None, None, logprob


# ---- the work that a call cannot do without

def work(c):
    if c["op"] == "verify":
        e, v = 4 if c["dtype"] == "f32" else 2, c["vocab"]
        rows = c["seqs"] * (c["drafts"] + 1)
        if c["ragged"]:
            u = torch.rand(c["seqs"], generator=torch.Generator().manual_seed(c["seqs"] * 31 + v)).tolist()
            counts = [min(1 + max(0, round(c["drafts"] * (1.2 * x - 0.1))), c["drafts"] + 1) for x in u]
            rows = c["drafts"] + 1 + sum(counts[1:])
        drafted = rows - c["seqs"] if c["model"] else 0
        # logits once; of the noise a row a sequence, where the entries are cut only a few
        return {"bytes": (rows + drafted) * v * e + (0 if c["cut"] else c["seqs"] * v * 4) + 20 * rows, "flops": 4 * (rows + drafted) * v}
    new, ctx = _lengths(c)
    tokens, e, d = sum(new), 2, c["d"]
    if c["op"] == "norm":
        elements = tokens * (c["hq"] + c["hkv"]) * d
        return {"bytes": tokens * (2 * (c["hq"] + 2 * c["hkv"]) * d * e + c["rot"] * 4 + 8) + 2 * d * e,
                "flops": 4 * elements + tokens * (c["hq"] + c["hkv"]) * c["rot"] * 3}
    lines = c["groups"] * c["prefix"] + tokens + sum(ctx)
    pairs = sum(n * (c["prefix"] + b) + n * (n + 1) // 2 for n, b in zip(new, ctx))
    return {"bytes": 2 * tokens * c["hq"] * d * e + tokens * c["hq"] * 4 + 2 * lines * c["hkv"] * d * e, "flops": 4 * pairs * c["hq"] * d}
