"""Verification of drafted tokens against the plain form in 64 bits.

p and q are exp(z) / sum in fp32: z of two roundings (2^-23 |z|), the exponential and the sum's logarithm some 2^-20, so with |z|
below 40 they are right to 1e-5.  A draft whose u q lies within 1e-4 of p, and two keys that lie closer than what p and q
leave open, are decisions that hang on a rounding: either answer passes there, and the test counts how few there are."""
import math

import pytest
import torch

import attn_ref as ref

pytestmark = pytest.mark.gpu
DT = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_09686_gb300 as pkg
    return pkg


class Batch:
    """Rows of logits of several sequences, drafts, numbers."""

    def __init__(self, drafts, v, dtype=torch.float32, model=True, seed=0, spread=2.0, likely=True):
        g = torch.Generator("cuda").manual_seed(seed * 31 + v)
        self.starts = [0]
        for d in drafts:
            self.starts.append(self.starts[-1] + d + 1 if d >= 0 else self.starts[-1])  # (-1: no rows at all)
        self.n, self.rows, self.v = len(drafts), self.starts[-1], v
        x = torch.randn(self.rows, v, device="cuda", generator=g) * spread
        self.logits = x.to(dtype)
        x = x + 0.5 * torch.randn(x.shape, device="cuda", generator=g)
        self.draft = x.to(dtype) if model else None
        self.noise = -torch.log(-torch.log(torch.rand(self.n, v, device="cuda", generator=g).clamp_(1e-10, 1 - 1e-7)))
        self.u = torch.rand(self.rows, device="cuda", generator=g)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.row_start = torch.tensor(self.starts, **i32)
        drawn = torch.softmax(x, -1).multinomial(1, generator=g)[:, 0] if likely else torch.randint(0, v, (self.rows,), device="cuda", generator=g)
        self.tokens = torch.cat((drawn[:1], drawn[:-1])).int()
        self.cuts, self.draft_cuts = {}, {}

    def set(self, which, **kw):
        i32 = dict(dtype=torch.int32, device="cuda")
        setattr(self, which, {k: torch.tensor(v, **i32) if k == "top_k" else torch.tensor(v, device="cuda") for k, v in kw.items()})
        return self

    def run(self, mf, logprob=True, stream=None, work=None):
        token = torch.full((self.rows,), -7, dtype=torch.int32, device="cuda")
        accepted = torch.full((self.n,), -7, dtype=torch.int32, device="cuda")
        lp = torch.full((self.rows,), 7.0, device="cuda") if logprob else None
        if work is None:
            work = torch.full((mf.mf_verify_bytes(self.n, self.rows, self.v),), 255, dtype=torch.uint8, device="cuda")
        mf.mf_verify(self.logits, self.row_start, self.tokens, self.u, self.noise, token, accepted, work, lp, mf.cuts(**self.cuts), self.draft,
                     mf.cuts(**self.draft_cuts), stream=stream)
        return token, accepted, lp

    def dist(self, row, s, draft):
        """(log p of the kept entries by index, z) of a row."""
        c = self.draft_cuts if draft else self.cuts

        def of(k, d):
            return c[k][s].item() if k in c else d
        kept, z = ref.kept64((self.draft if draft else self.logits)[row].float(), of("temperature", 1.0), of("top_k", 0), of("top_p", 1.0),
                             of("min_p", 0.0))
        if not kept:
            return {}
        total = math.log(math.fsum(math.exp(z[i]) for i in kept))
        return {i: z[i] - total for i in kept}

    def check(self, mf, close_allowed=None):
        token, accepted, lp = (x.tolist() for x in self.run(mf))
        u, tokens, close = self.u.double().tolist(), self.tokens.tolist(), 0
        for s in range(self.n):
            b, e = self.starts[s], self.starts[s + 1]
            if b == e:
                assert accepted[s] == 0
                continue
            taken, open_ = 0, False
            for row in range(b, e):
                p = self.dist(row, s, False)
                q, x = {}, None
                if row + 1 < e:
                    x = tokens[row + 1]
                    q = self.dist(row, s, True) if self.draft is not None else {x: 0.0}
                    px, qx = math.exp(p.get(x, -math.inf)), math.exp(q.get(x, -math.inf))
                    if px > 0 and abs(u[row] * qx - px) <= 1e-4 * px:  # (0 is 0 on either side)
                        close += 1
                        open_ = True
                        break
                    if u[row] * qx < px:
                        assert token[row] == x and abs(lp[row] - p[x]) <= 2e-5 * max(1.0, abs(p[x])), (s, row)
                        taken += 1
                        continue
                g = self.noise[s].double().nan_to_num(-math.inf, math.inf, -math.inf).tolist()
                keys = []
                for i, v in p.items():
                    w = math.exp(q[i]) if i in q else 0.0
                    left = math.exp(v) - w
                    if left > 0:
                        keys.append((math.log(left) + g[i], -i, 2e-5 * (math.exp(v) + w) / left + 1e-6 * abs(g[i])))
                if not keys:
                    keys = [(v + g[i], -i, 2e-5) for i, v in p.items()]
                keys.sort(reverse=True)
                if not keys:
                    assert token[row] == -1 and lp[row] == -math.inf
                    break
                near = [-k[1] for k in keys if k[0] >= keys[0][0] - k[2] - keys[0][2]] if math.isfinite(keys[0][0]) else [-keys[0][1]]
                close += len(near) > 1
                assert token[row] in near, (s, row, token[row], near[:4])
                assert abs(lp[row] - p[token[row]]) <= 2e-5 * max(1.0, abs(p[token[row]]))
                break
            if open_:
                continue
            assert accepted[s] == taken, (s, accepted[s], taken)
            assert all(t == -1 for t in token[b + taken + 1:e]) and all(v == -math.inf for v in lp[b + taken + 1:e])
        assert close <= (1 + self.rows // 50 if close_allowed is None else close_allowed)
        return token, accepted, lp


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("v", [1, 2, 31, 1000, 5003])
@pytest.mark.parametrize("model", [True, False])
def test_by_temperature(mf, dtype, v, model):
    b = Batch([4, 0, 1, 7, 3, 2, 5], v, dtype, model)
    b.check(mf, 50 if v <= 2 else None)
    t = [0.7, 1.3, 1.0, 0.5, 2.0, 1.0, 0.9]
    b.set("cuts", temperature=t).set("draft_cuts", temperature=t[::-1]).check(mf, 50 if v <= 2 else None)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("v", [50001, 131072])
@pytest.mark.parametrize("model", [True, False])
def test_large_vocabularies(mf, dtype, v, model):
    b = Batch([2, 1], v, dtype, model)
    b.check(mf)
    b.set("cuts", temperature=[0.7, 1.0], top_k=[50, 0], top_p=[0.9, 0.95]).set("draft_cuts", temperature=[0.7, 1.0], min_p=[0.05, 0.001])
    b.check(mf)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("model", [True, False])
def test_all_cuts(mf, dtype, model):
    b = Batch([3, 1, 0, 6, 4, 2, 3, 8], 3001, dtype, model)
    both = dict(temperature=[0.7, 1.0, 0.0, 1.3, 0.6, 1.0, 2.0, 1.0], top_k=[0, 50, 7, 1000, 2500, 1, 0, 20],
                top_p=[1.0, 0.9, 0.5, 0.8, 0.99, 1.0, 0.0, 0.95], min_p=[0.0, 0.02, 0.3, 0.0, 0.001, 0.0, 0.0, 1.5])
    b.set("cuts", **both).check(mf)
    b.set("draft_cuts", **both).check(mf)
    b.set("cuts", temperature=both["temperature"]).check(mf)


@pytest.mark.parametrize("model", [True, False])
def test_u_at_its_ends(mf, model):
    """u = 0 takes whatever has any probability, u just below 1 takes where the drafter was no surer than the target."""
    b = Batch([6, 6], 300, torch.float32, model)
    b.u.zero_()
    assert b.check(mf, 20)[1] == [6, 6]
    b.u.fill_(1 - 2.0 ** -24)
    b.check(mf)
    b.u.fill_(math.nan)
    assert b.run(mf)[1].tolist() == [0, 0]


@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("dtype", DT)
def test_a_drafter_that_is_the_target(mf, cut, dtype):
    """Equal rows and settings: every draft is taken, whatever u below 1; the last token is what sampling gives."""
    b = Batch([6, 0, 12], 5003, dtype)
    b.draft = b.logits.clone()
    if cut:
        kw = dict(temperature=[0.8, 1.0, 1.2], top_k=[0, 40, 0], top_p=[0.9, 1.0, 0.8], min_p=[0.0, 0.01, 0.0])
        b.set("cuts", **kw).set("draft_cuts", **kw)
        for s in range(3):  # drafts that the drafter can have drawn
            for row in range(b.starts[s], b.starts[s + 1] - 1):
                b.tokens[row + 1] = max(b.dist(row, s, True).items(), key=lambda e: e[1] + b.noise[s, e[0]].item())[0]
    b.u.fill_(1 - 2.0 ** -24)
    token, accepted, lp = b.run(mf)
    assert accepted.tolist() == [6, 0, 12]
    last = b.row_start[1:].long() - 1
    want, wlp = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda")
    mf.mf_sample(b.logits[last], b.noise, want, wlp, **b.cuts)
    assert torch.equal(token[last], want) and (lp[last] - wlp).abs().max() < 2e-5


def test_equal_rows_and_a_draft_that_is_not_taken(mf):
    """No entry has p > q: the token comes from p itself."""
    b = Batch([2], 50)
    b.draft = b.logits.clone()
    b.u.fill_(1.5)  # (outside [0, 1): refuses all)
    token, accepted, _ = b.run(mf)
    key = torch.log_softmax(b.logits[0].double(), 0) + b.noise[0]
    assert accepted.tolist() == [0] and token.tolist() == [int(key.argmax()), -1, -1]


@pytest.mark.parametrize("model", [True, False])
def test_drafts_outside_the_vocabulary(mf, model):
    b = Batch([3, 2, 1], 100, torch.float32, model)
    b.u.zero_()
    b.tokens[2], b.tokens[5], b.tokens[8] = -1, 100, 2 ** 31 - 1
    token, accepted, lp = b.check(mf)
    assert accepted == [1, 0, 1] or not model or accepted[1] == 0


def test_rows_of_infinities_and_nan(mf):
    b = Batch([2, 2, 2, 2, 1], 200, torch.float32)
    b.logits[0] = -math.inf                      # nothing is allowed
    b.logits[3] = math.nan
    b.logits[6, 17] = b.logits[6, 90] = math.inf  # two entries share the mass
    b.logits[9, ::2] = -math.inf
    b.logits[9, 1::4] = math.nan
    b.draft[9, 40:] = -math.inf
    b.draft[12] = -math.inf                      # a drafter that could have drawn nothing
    b.noise[3, :50] = math.nan
    token, accepted, lp = b.check(mf)
    assert token[0] == token[3] == -1 and token[6] in (17, 90) and abs(lp[6] + math.log(2)) < 1e-5


def test_greedy(mf):
    """Temperature 0 on both sides: drafts are taken while they are the target's first choice, ties to the lower index."""
    b = Batch([3, 3, 3], 500, torch.bfloat16, likely=False)
    b.logits[4, 7] = b.logits[4, 3] = 50
    b.set("cuts", temperature=[0.0] * 3).set("draft_cuts", temperature=[0.0] * 3)
    best = b.logits.float().argmax(-1)
    for row in (0, 1, 4, 8, 9, 10):
        b.tokens[row + 1] = 3 if row == 4 else best[row]
    for b.draft in (b.logits.clone(), None):
        token, accepted, lp = b.run(mf)
        assert accepted.tolist() == [2, 1, 3]
        assert token.tolist() == [int(best[0]), int(best[1]), int(best[2]), -1, 3, int(best[5]), -1, -1] + [int(x) for x in best[8:]]
        assert (lp[token >= 0] == 0).all()


def test_many_drafts(mf):
    """More drafts than a block has threads."""
    b = Batch([700, 1300], 20, torch.float32)
    b.draft = b.logits.clone()
    token, accepted, _ = b.run(mf)
    assert accepted.tolist() == [700, 1300]
    b.u[650], b.u[701 + 1299] = 1.5, 1.5
    token, accepted, _ = b.run(mf)
    assert accepted.tolist() == [650, 1299] and (token[651:701] == -1).all() and token[700 + 1 + 1300] == -1


def test_sequences_without_rows_and_rows_of_nobody(mf):
    b = Batch([-1, 2, -1, -1, 0, 3, -1], 300)
    token, accepted, lp = b.check(mf)
    wide = Batch([3, 3], 300)
    wide.row_start = torch.tensor([2, 4, 7], dtype=torch.int32, device="cuda")
    token, accepted, lp = wide.run(mf)
    assert (token[:2] == -7).all() and (token[7:] == -7).all() and (lp[:2] == 7).all() and (lp[7:] == 7).all() and (token[2:7] != -7).all()


@pytest.mark.parametrize("starts", [[-5, 4, 900], [4, 2, 8], [8, 8, 8], [0, 2 ** 31 - 1, -2 ** 31], [900, 901, 902]])
def test_row_starts_out_of_range(mf, starts):
    """Taken as the nearest valid ones: nothing outside is touched, and sequences whose rows are in order are right."""
    b = Batch([3, 3], 300)
    b.row_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    token, accepted, lp = b.run(mf)
    ends = [min(max(x, 0), 8) for x in starts]
    for s in range(2):
        rows = max(ends[s + 1] - ends[s], 0)
        assert 0 <= accepted[s].item() <= max(rows - 1, 0)
    assert all(-7 <= t < 300 for t in token.tolist())


@pytest.mark.parametrize("dtype", DT)
def test_views_of_any_alignment(mf, dtype):
    want = Batch([3, 1, 4], 1001, dtype)
    a = want.run(mf)
    for pad, off in ((1, 0), (7, 3), (5, 5)):
        def view(x):
            big = torch.full((x.shape[0], x.shape[1] + pad + off), math.nan, dtype=x.dtype, device="cuda")
            big[:, off:off + x.shape[1]] = x
            return big[:, off:off + x.shape[1]]
        b = Batch([3, 1, 4], 1001, dtype)
        b.logits, b.draft, b.noise = view(b.logits), view(b.draft), view(b.noise)
        token, accepted, lp = b.run(mf)
        assert torch.equal(token, a[0]) and torch.equal(accepted, a[1])
        # the order of a row's sum follows its alignment: two trees of 1001 terms, some 20 levels of 2^-24 each
        assert ((lp - a[2]).abs() <= 40 * 2.0 ** -24 + 2.0 ** -22 * lp.abs()).logical_or(lp == a[2]).all()


def test_largest_vocabulary(mf):
    v = 1 << 20
    b = Batch([1, 2], v, torch.bfloat16)
    b.draft = b.logits.clone()
    token, accepted, lp = b.run(mf)
    assert accepted.tolist() == [1, 2]
    for s, row in ((0, 1), (1, 4)):
        lpd = torch.log_softmax(b.logits[row].double(), 0)
        key = (lpd + b.noise[s]).topk(2)
        assert key.values[0] - key.values[1] < 1e-4 or token[row] == key.indices[0]
        assert abs(lp[row].item() - lpd[token[row].long()].item()) < 2e-5 * 20


@pytest.mark.parametrize("model", [True, False])
@pytest.mark.parametrize("cut", [False, True])
def test_the_tokens_are_the_targets_draws(mf, model, cut):
    """20000 sequences of one draft: the first token's frequencies are p's (each within six of its standard deviations)."""
    n, v = 20000, 12
    g = torch.Generator("cuda").manual_seed(3)
    b = Batch([1] * n, v, torch.float32, model)
    b.logits.copy_(torch.randn(2, v, device="cuda", generator=g).repeat(n, 1))
    kw = dict(temperature=[0.8] * n, top_k=[7] * n, top_p=[0.9] * n) if cut else dict(temperature=[0.8] * n)
    b.set("cuts", **kw).set("draft_cuts", temperature=[1.1] * n)
    if model:
        b.draft.copy_(torch.randn(2, v, device="cuda", generator=g).repeat(n, 1))
        drawn = torch.softmax(b.draft[::2] / 1.1, -1).multinomial(1, generator=g)[:, 0]
    else:
        drawn = torch.randint(0, v, (n,), device="cuda", generator=g)
    b.tokens[1::2] = drawn.int()
    token, accepted, lp = b.run(mf)
    p = torch.zeros(v, dtype=torch.float64)
    for i, x in b.dist(0, 0, False).items():
        p[i] = math.exp(x)
    seen = torch.bincount(token[::2].long().cpu(), minlength=v).double()
    assert ((seen - n * p).abs() <= 6 * torch.sqrt(n * p * (1 - p)) + 1e-9).all(), (seen, n * p)


def test_streams_graphs_and_workspaces(mf):
    """Two calls at once on streams and workspaces of their own, a captured one replayed with other inputs, the same bits again."""
    a, b = Batch([4, 2, 0], 5003, torch.bfloat16), Batch([3, 3, 1], 5003, torch.bfloat16, seed=4)
    want = [x.run(mf) for x in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = []
        for x, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                got.append(x.run(mf))
        torch.cuda.synchronize()
        for x, y in zip(want, got):
            assert all(torch.equal(p, q) for p, q in zip(x, y))
    s = streams[0]
    work = torch.empty(mf.mf_verify_bytes(3, a.rows, 5003), dtype=torch.uint8, device="cuda")
    with torch.cuda.stream(s):
        a.logits.add_(0)
        out = a.run(mf, work=work)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            out = a.run(mf, work=work)
        for seed in (8, 9):
            o = Batch([4, 2, 0], 5003, torch.bfloat16, seed=seed)
            for name in ("logits", "draft", "noise", "u", "tokens"):
                getattr(a, name).copy_(getattr(o, name))
            g.replay()
            s.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(out, o.run(mf)))


def test_copies_that_do_not_arrive(mf):
    """The answer is the same when the rows' copies into shared memory come too late (as in sampling)."""
    b = Batch([2, 1], 3001, torch.bfloat16).set("cuts", top_p=[0.9, 0.8], top_k=[0, 40])
    want = b.run(mf)
    mf.mf_sample_test_hold(1)
    try:
        got = b.run(mf)
    finally:
        mf.mf_sample_test_hold(0)
    assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_tensors_that_do_not_fit_are_refused(mf):
    b = Batch([2, 1], 300)
    i32 = dict(dtype=torch.int32, device="cuda")
    good = dict(logits=b.logits, row_start=b.row_start, tokens=b.tokens, u=b.u, noise=b.noise, token=torch.empty(5, **i32),
                accepted=torch.empty(2, **i32), work=torch.empty(mf.mf_verify_bytes(2, 5, 300), dtype=torch.uint8, device="cuda"),
                logprob=torch.empty(5, device="cuda"), draft_logits=b.draft)
    short = mf.cuts(temperature=torch.ones(1, device="cuda"))

    def refused(**kw):
        with pytest.raises(mf.MFError) as e:
            mf.mf_verify(**{**good, **kw})
        assert e.value.status == mf.MF_E_INVAL

    for t in (b.logits.double(), b.logits[:, :299], b.logits[:, ::2], b.logits[0], b.logits.cpu(), b.logits.half()):
        refused(logits=t)
    for t in (b.draft.half(), b.draft[:4], b.draft[:, :299], b.draft.cpu(), b.draft.t().contiguous().t()):
        refused(draft_logits=t)
    for t in (b.noise.half(), b.noise[:, :299], b.noise[0], b.noise.cpu()):
        refused(noise=t)
    for name, n in (("row_start", 3), ("tokens", 5), ("u", 5), ("token", 5), ("accepted", 2), ("logprob", 5)):
        t = good[name]
        for bad in (t[:n - 1], t.double(), t.cpu(), t.repeat(2)[::2]):
            refused(**{name: bad})
    refused(work=good["work"][:-16])
    refused(work=good["work"].cpu())
    refused(cuts=short)
    refused(draft_cuts=short)
    mf.mf_verify(**good)
    torch.cuda.synchronize()


def by_the_formula(b, token, accepted, lp):
    """Rows that are not cut against the formula, by torch in 64 bits (check() for large vocabularies): the number that refused a draft.  A key
    is right to 2e-5 of p + q over p - q and 1e-6 of the noise (see above): the one that is taken may lie below the largest by both keys'
    part of that."""
    refused = close = 0
    for s in range(b.n):
        for row in range(b.starts[s], b.starts[s + 1]):
            p, q, t = torch.softmax(b.logits[row].double(), 0), None, int(token[row])
            last = row + 1 == b.starts[s + 1]
            if not last:
                x = int(b.tokens[row + 1])
                if b.draft is None:
                    q = torch.zeros_like(p)
                    q[x] = 1
                else:
                    q = torch.softmax(b.draft[row].double(), 0)
                uq, px = float(b.u[row]) * float(q[x]), float(p[x])
                if abs(uq - px) <= 1e-4 * px:  # (hangs on a rounding: either answer, and nothing is said of what follows)
                    close += 1
                    break
                if uq < px:
                    assert t == x and abs(float(lp[row]) - math.log(px)) <= 2e-5 * max(1.0, abs(math.log(px)))
                    continue
                refused += 1
            rest, g = p if last else p - q, b.noise[s].double()
            some, safe = rest > 0, rest.clamp_min(1e-300)
            key = torch.where(some, safe.log() + g, -math.inf)
            off = torch.where(some, 2e-5 * (p if last else p + q) / safe + 1e-6 * g.abs(), 0.0)
            best = int(key.argmax())
            assert some[t] and key[t] >= key[best] - off[t] - off[best], (s, row, t, best)
            assert abs(float(lp[row]) - float(p[t].log())) <= 2e-5 * max(1.0, abs(float(p[t].log())))
            assert int(accepted[s]) == row - b.starts[s] and (token[row + 1:b.starts[s + 1]] == -1).all()
            break
    assert close <= 1 + b.rows // 50
    return refused


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("model", [True, False])
def test_copies_of_more_chunks_than_the_ring_holds_that_do_not_arrive(mf, model, dtype):
    """Nothing is cut, so that only the pass over the deciding row copies: 16 chunks a block, 8 stages.  Stages whose copies were given up are
    not filled again."""
    b = Batch([1, 2], 1 << 18, dtype, model)
    b.u.fill_(1.5)
    want = b.run(mf)
    assert by_the_formula(b, *want) > 0
    mf.mf_sample_test_hold(1)
    try:
        got = b.run(mf)
        torch.cuda.synchronize()
    finally:
        mf.mf_sample_test_hold(0)
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    assert all(torch.equal(p, q) for p, q in zip(want, b.run(mf)))


def as_if_rising(starts, rows):
    """Starts inside the rows, each the largest so far."""
    at, out = 0, []
    for x in starts:
        at = max(at, min(max(x, 0), rows))
        out.append(at)
    return out


@pytest.mark.parametrize("cut", [(), ("cuts",), ("draft_cuts",), ("cuts", "draft_cuts")])
@pytest.mark.parametrize("starts", [[0, 5, 3, 4], [0, 5, 3, 11], [4, 2, 8, 12], [0, 2 ** 31 - 1, -2 ** 31, 6], [3, 0, 0, 12],
                                    [2, 6, 6, 5, 1, 9], [5, 4, 3, 2, 1]])
def test_row_starts_that_fall(mf, starts, cut):
    """Taken as the largest so far: a row has one sequence, whose settings and numbers it goes by; the others are not touched."""
    n = len(starts) - 1
    b = Batch([11] + [-1] * (n - 1), 300, torch.bfloat16)
    for which in cut:
        b.set(which, temperature=[0.7 + 0.1 * s for s in range(n)], top_k=[50 - 9 * s for s in range(n)], top_p=[0.9 - 0.05 * s for s in range(n)])
    b.starts, b.row_start = as_if_rising(starts, b.rows), torch.tensor(starts, dtype=torch.int32, device="cuda")
    token, accepted, lp = b.check(mf)
    for row in list(range(b.starts[0])) + list(range(b.starts[-1], b.rows)):
        assert token[row] == -7 and lp[row] == 7


@pytest.mark.parametrize("cut", [False, True])
def test_row_starts_of_many_sequences_that_fall(mf, cut):
    """More sequences than are listed in shared memory, some of whose starts lie below earlier ones."""
    n = 2500
    b = Batch([1] * n, 9, torch.float32)
    starts = list(b.starts)
    for s in (3, 700, 701, 2300, n):
        starts[s] -= 300
    if cut:
        b.set("cuts", temperature=[0.5 + 0.5 * (s % 3) for s in range(n)], top_k=[9 - s % 8 for s in range(n)])
    b.starts, b.row_start = as_if_rising(starts, b.rows), torch.tensor(starts, dtype=torch.int32, device="cuda")
    b.check(mf)


@pytest.mark.parametrize("dtype,drafts", [(torch.float32, [1, 2]), (torch.bfloat16, [3]), (torch.float16, [0, 1, 1])])
@pytest.mark.parametrize("model", [True, False])
def test_refused_drafts_of_the_largest_vocabulary(mf, dtype, drafts, model):
    """64 chunks a block (C = 8), the ring's stages used again and again, with the drafter's rows and without; u above 1 refuses nearly all."""
    b = Batch([d for d in drafts if d], 1 << 20, dtype, model, seed=2)
    b.u.fill_(1.5)
    assert by_the_formula(b, *b.run(mf)) > 0


@pytest.mark.parametrize("seqs,v", [(64, 131072), (130, 50001), (48, 200001), (210, 40003)])
@pytest.mark.parametrize("dtype,model", [(torch.bfloat16, True), (torch.float16, True), (torch.float32, True), (torch.bfloat16, False)])
def test_refused_drafts_of_many_sequences(mf, seqs, v, dtype, model):
    """Clusters of fewer blocks, several blocks an SM and rings of fewer stages."""
    b = Batch([1 + s % 2 for s in range(seqs)], v, dtype, model, seed=3)
    b.u.fill_(1.5)
    assert by_the_formula(b, *b.run(mf)) > 0


@pytest.mark.parametrize("model", [True, False])
def test_drafts_that_no_vocabulary_has(mf, model):
    """u = 0 takes every draft that can be, up to the one that is no token: what is taken there, and what ends the rows, to the number."""
    b = Batch([3, 2, 1], 100, torch.float32, model)
    b.u.zero_()
    b.tokens[2], b.tokens[5], b.tokens[8] = -1, 100, 2 ** 31 - 1
    token, accepted, lp = b.check(mf)
    assert accepted == [1, 0, 0]
    assert token[0] == b.tokens[1] and token[2:4] == [-1, -1] and token[5:7] == [-1, -1] and token[8] == -1
    assert all(0 <= token[row] < 100 for row in (1, 4, 7))
