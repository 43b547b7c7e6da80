"""The paged attention, the append with rotation and the sampling written out plainly in 64 bits, and cases of them."""
import math

import torch

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # unit roundoff


class Case:
    """A cache with garbage wherever no line of a sequence lies, and a step over it."""

    def __init__(self, new, ctx, hq=8, hkv=2, d=64, dtype="bf16", page=16, heads_first=False, seed=0, spare=2,
                 garbage=math.nan, row_pad=0, base_page=0):
        g = torch.Generator("cuda").manual_seed(seed + 1)
        self.new, self.len = list(new), [a + b for a, b in zip(new, ctx)]
        self.hq, self.hkv, self.d, self.page, self.dtype = hq, hkv, d, page, dtype
        n = len(self.new)
        need = [-(-t // page) for t in self.len]
        pool = sum(need) + spare
        order = (torch.randperm(pool, device="cuda", generator=g) + base_page).tolist()
        width = max(1, max(need))
        table = torch.full((n, width), base_page, dtype=torch.int32)
        shape = (pool + base_page, hkv, page, d) if heads_first else (pool + base_page, page, hkv, d)
        self.k, self.v = (torch.empty(shape, dtype=DT[dtype], device="cuda") for _ in range(2))
        if heads_first:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        for c in (self.k, self.v):
            c[base_page:] = garbage
        self.lines = []  # (pages, lines in them) of each sequence's positions
        at = 0
        for s in range(n):
            mine = order[at:at + need[s]]
            at += need[s]
            table[s, :need[s]] = torch.tensor(mine, dtype=torch.int32)
            pos = torch.arange(self.len[s])
            pg = torch.tensor(mine, dtype=torch.long)[pos // page] if need[s] else torch.zeros(0, dtype=torch.long)
            self.lines.append((pg.cuda(), (pos % page).cuda()))
            for c in (self.k, self.v):
                c[self.lines[s][0], self.lines[s][1]] = torch.randn(self.len[s], hkv, d, device="cuda", generator=g).to(c.dtype)
        starts = [0]
        for x in self.new:
            starts.append(starts[-1] + x)
        self.start, self.tokens, self.max_q = starts, starts[-1], max(1, max(self.new))
        self.q_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.kv_len = torch.tensor(self.len, dtype=torch.int32, device="cuda")
        self.pages = table.cuda()
        rows = torch.randn(self.tokens, (hq + 2 * hkv) * d + row_pad, device="cuda", generator=g).to(DT[dtype])
        self.q = rows[:, :hq * d].unflatten(1, (hq, d))
        self.new_k = rows[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
        self.new_v = rows[:, (hq + hkv) * d:(hq + 2 * hkv) * d].unflatten(1, (hkv, d))

    def step(self, mf, **kw):
        return mf.step(kw.get("q_start", self.q_start), self.kv_len, self.pages, self.tokens, self.max_q)

    def attn(self, mf):
        shape = mf.AttnShape(self.hq, self.hkv, self.d, mf.MF_BF16 if self.dtype == "bf16" else mf.MF_F16)
        return mf.mf_attn_create(shape, len(self.new), max(1, self.tokens), 0)


def attention64(c, scale, window=0, causal=True):
    """(out, lse, tolerance of out, tolerance of lse) in 64 bits.

    Tolerance: the probabilities and the output are each rounded to the dtype once (u sum p |v| and u |o|; in fp16 a
    probability may also fall below the normal range: half its smallest step, 2^-25, each, against a sum of at
    least 1); a score's fp32 error is at most (d + 2) 2^-24 sum |q k| scale, that of exp and the sums a few 2^-22 and
    (n + 4) 2^-24 for n lines, all relative to p.  lse: the score's error plus the sum's, plus its own rounding."""
    u = U[c.dtype]
    out = torch.zeros(c.tokens, c.hq, c.d, dtype=torch.float64, device="cuda")
    tol, lse = torch.zeros_like(out), torch.full((c.tokens, c.hq), -math.inf, dtype=torch.float64, device="cuda")
    ltol = torch.zeros_like(lse)
    for s, n in enumerate(c.len):
        lo = max(0, n - c.new[s] - window + 1) if window else 0  # lines before it may hold anything
        k, v = (x[c.lines[s][0][lo:], c.lines[s][1][lo:]].double() for x in (c.k, c.v))
        line = torch.arange(lo, n, device="cuda")
        for i0 in range(0, c.new[s] if n else 0, 256):
            i1 = min(i0 + 256, c.new[s])
            t = slice(c.start[s] + i0, c.start[s] + i1)
            pos = torch.arange(n - c.new[s] + i0, n - c.new[s] + i1, device="cuda")[:, None]
            see = torch.ones(i1 - i0, n - lo, dtype=torch.bool, device="cuda")
            if window:
                see &= line > pos - window
            if causal:
                see &= line <= pos
            num = see.sum(-1).double()[:, None, None]
            q = c.q[t].double().unflatten(1, (c.hkv, c.hq // c.hkv))
            x = torch.einsum("thgd,jhd->thgj", q, k) * scale
            mag = (torch.einsum("thgd,jhd->thgj", q.abs(), k.abs()) * abs(scale)).masked_fill_(~see[:, None, None], 0)
            x.masked_fill_(~see[:, None, None], -math.inf)
            z = torch.logsumexp(x, -1)
            p = torch.exp(x - torch.where(z.isinf(), 0.0, z)[..., None])
            o = torch.einsum("thgj,jhd->thgd", p, v)
            rel = (c.d + 2) * 2.0 ** -24 * mag.amax(-1) + (num + 4) * 2.0 ** -24 + 2.0 ** -20
            size = torch.einsum("thgj,jhd->thgd", p, v.abs())
            tiny = num[..., None] * 2.0 ** -25 * v.abs().amax() if c.dtype == "f16" else 0.0
            out[t], lse[t] = o.flatten(1, 2), z.flatten(1, 2)
            tol[t] = (u * (size + o.abs()) * 1.01 + 3 * rel[..., None] * size + tiny + 2.0 ** -24).flatten(1, 2)
            ltol[t] = (2 * rel + 2.0 ** -22 * z.abs()).flatten(1, 2).nan_to_num(0)
    return out, lse, tol, ltol


def rotate64(x, cos, sin, interleaved):
    """x [T][heads][d], cos and sin [T][pairs]: the rotated copy, and the sum of the magnitudes of each result's terms."""
    y, size = x.double().clone(), x.double().abs()
    half = cos.shape[1]
    for j in range(half):
        i0, i1 = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        a, b, co, si = x[..., i0].double(), x[..., i1].double(), cos[:, j:j + 1].double(), sin[:, j:j + 1].double()
        y[..., i0], y[..., i1] = a * co - b * si, b * co + a * si
        size[..., i0], size[..., i1] = (a * co).abs() + (b * si).abs(), (b * co).abs() + (a * si).abs()
    return y, size


def kept64(x, t, k, p, mp):
    """The kept entries of one row (a list of indices in order), and z, in 64 bits."""
    x = [(-math.inf if v != v else float(v)) for v in x.tolist()]
    order = sorted((i for i in range(len(x)) if x[i] > -math.inf), key=lambda i: -x[i])
    if not order:
        return [], {}
    m = x[order[0]]
    greedy = not t > 0
    z = {i: (0.0 if x[i] == m else (x[i] - m) / (1.0 if greedy else t)) for i in order}
    if greedy:
        return order[:1], z
    if k > 0:
        order = order[:k]
    w = [math.exp(z[i]) for i in order]
    total, before, n = math.fsum(w), 0.0, 0
    for wi in w:
        if n and p < 1 and not before < p * total:
            break
        n += 1
        before += wi
    return [i for r, i in enumerate(order[:n]) if r == 0 or w[r] >= min(mp, 1.0)], z
