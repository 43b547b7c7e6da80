"""Sampling against the plain form in 64 bits.

Inputs are such that no decision hangs on a rounding: borders of top-p lie between the mass of whole entries by more than
1e-4 of the total, and the noise is drawn, so that two keys are never within 1e-4 of the best (the
test checks this of its inputs before it compares)."""
import math

import pytest
import torch

import attn_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_09686_gb300 as pkg
    return pkg


def gumbel(n, v, seed=0):
    g = torch.Generator("cuda").manual_seed(seed + 99)
    return -torch.log(-torch.log(torch.rand(n, v, device="cuda", generator=g).clamp_(1e-10, 1 - 1e-7)))


def run(mf, x, noise, t=None, k=None, p=None, mp=None, logprob=True):
    n = x.shape[0]

    def vec(v, dt=torch.float32):
        return None if v is None else torch.tensor([v] * n if not isinstance(v, list) else v, dtype=dt, device="cuda")

    token = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((n,), 7.0, device="cuda") if logprob else None
    mf.mf_sample(x, noise, token, lp, vec(t), vec(k, torch.int32), vec(p), vec(mp))
    return token.tolist(), lp.tolist() if logprob else None


def check(mf, x, noise, t=None, k=None, p=None, mp=None):
    got, lp = run(mf, x, noise, t, k, p, mp)
    close = 0
    for r in range(x.shape[0]):
        def of(v, d):
            return d if v is None else v[r] if isinstance(v, list) else v
        kept, z = ref.kept64(x[r].float(), of(t, 1.0), of(k, 0), torch.tensor(of(p, 1.0)).item(), torch.tensor(of(mp, 0.0)).item())
        if not kept:
            assert got[r] == -1 and lp[r] == -math.inf
            continue
        g = noise[r].double().nan_to_num(-math.inf, math.inf, -math.inf).tolist()
        key = sorted(((z[i] + g[i], -i) for i in kept), reverse=True)
        if len(key) > 1 and key[0][0] - key[1][0] < 1e-4 * max(1.0, abs(key[0][0])) and key[0][0] != key[1][0]:
            close += 1
            assert got[r] in (-key[0][1], -key[1][1])
            continue
        assert got[r] == -key[0][1], (r, got[r], -key[0][1])
        # the fp32 z and the sum's relative error (2^-20 covers exp and a tree over 2^20 entries)
        want = z[got[r]] - math.log(math.fsum(math.exp(z[i]) for i in kept))
        assert abs(lp[r] - want) <= 2.0 ** -22 * abs(z[got[r]]) + 2.0 ** -20 + 2.0 ** -23 * abs(want)
    assert close <= 1 + x.shape[0] // 50
    return got


DT = [torch.float32, torch.float16, torch.bfloat16]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("v", [1, 2, 31, 1000, 4096, 50001, 131072, 262147])
def test_temperature_alone(mf, dtype, v):
    g = torch.Generator("cuda").manual_seed(v)
    x = (torch.randn(3, v, device="cuda", generator=g) * 3).to(dtype)
    check(mf, x, gumbel(3, v, v), t=[1.0, 0.5, 1.7])


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("v", [1, 7, 1000, 50001, 262147])
def test_top_k(mf, dtype, v):
    g = torch.Generator("cuda").manual_seed(v + 1)
    ks = [1, 2, 3, 20, 50, 1000, 5000, v - 1, v, v + 5, 0, -1]
    x = (torch.randn(len(ks), v, device="cuda", generator=g) * 3).to(dtype)
    check(mf, x, gumbel(len(ks), v, v), k=ks)


def spaced(v, n, seed, ratio, dtype=torch.float32):
    """Rows whose sorted probabilities fall by a fixed ratio: running masses are known and well apart."""
    g = torch.Generator("cuda").manual_seed(seed)
    perm = torch.stack([torch.randperm(v, device="cuda", generator=g) for _ in range(n)])
    return (torch.arange(v, device="cuda").float()[perm] * math.log(ratio)).to(dtype)


@pytest.mark.parametrize("v", [3, 1000, 50001])
@pytest.mark.parametrize("ratio", [0.5, 0.9, 0.99])
def test_top_p(mf, v, ratio):
    ps = [0.0, -1.0, 0.3, 0.505, 0.9003, 0.95007, 1.0, 2.0, math.nan]
    x = spaced(v, len(ps), v, ratio)
    noise = gumbel(len(ps), v, v)
    check(mf, x, noise, p=[1.0 if p != p else p for p in ps])
    a, b = (run(mf, x, noise, p=q) for q in (ps, [1.0 if p != p else p for p in ps]))
    assert a == b


@pytest.mark.parametrize("v", [3, 1000, 50001])
def test_min_p(mf, v):
    ms = [0.0, -1.0, 0.0503, 0.5003, 1.0, 3.0]
    x = spaced(v, len(ms), v, 0.9)
    check(mf, x, gumbel(len(ms), v, v), mp=ms)


@pytest.mark.parametrize("dtype", DT)
def test_all_together(mf, dtype):
    n, v = 40, 5003
    g = torch.Generator("cuda").manual_seed(5)
    x = (torch.randn(n, v, device="cuda", generator=g) * 2).to(dtype)
    check(mf, x, gumbel(n, v), t=[0.7, 1.0, 0.0, 1.3] * 10, k=[0, 50, 7, 1000, 4000] * 8, p=[1.0, 0.9, 0.5003, 0.8] * 10,
          mp=[0.0, 0.02, 0.3] * 13 + [0.0])


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("v", [40, 3001, 70000])
def test_ties(mf, dtype, v):
    """Few distinct values: the border falls among equal ones, which count in the order of their index."""
    g = torch.Generator("cuda").manual_seed(v)
    ks = [1, 2, 5, 17, 100, v // 3, v // 2 + 1, v - 1]
    x = torch.randint(0, 4, (len(ks), v), device="cuda", generator=g).float().mul_(0.5).to(dtype)
    check(mf, x, gumbel(len(ks), v), k=ks)
    one = torch.zeros(len(ks), v, device="cuda", dtype=dtype)
    check(mf, one, gumbel(len(ks), v, 3), k=ks)
    # of equal entries top-p keeps the first ceil(p v)
    p = [(j + 0.5) / v for j in (0, 1, 5, v // 2, v - 2)]
    check(mf, one[:5], gumbel(5, v, 4), p=p)


def test_greedy_takes_the_lowest_of_the_largest(mf):
    x = torch.randn(6, 3000, device="cuda")
    x[:, 700] = x[:, 699] = x[:, 2999] = 9.0
    for t in (0.0, -1.0, math.nan):
        got, lp = run(mf, x, gumbel(6, 3000), t=t, k=50, p=0.5, mp=0.1)
        assert got == [699] * 6 and lp == [0.0] * 6


@pytest.mark.parametrize("dtype", DT)
def test_masked_rows(mf, dtype):
    """Forbidden entries of -inf, NaN or the type's lowest value, rows of nothing else, +inf."""
    n, v = 8, 2050
    g = torch.Generator("cuda").manual_seed(8)
    x = (torch.randn(n, v, device="cuda", generator=g) * 2).to(dtype)
    x[0, ::2] = -math.inf
    x[1] = -math.inf
    x[2] = math.nan
    x[3, 5:] = math.nan
    x[4, 3:] = torch.finfo(dtype).min
    x[5] = torch.finfo(dtype).min
    x[6, 77] = math.inf
    x[7, 10:40:3] = math.inf
    noise = gumbel(n, v)
    noise[0, 1:200:2] = math.nan
    for kw in (dict(), dict(k=3), dict(p=0.9003), dict(mp=0.3003), dict(t=0.0), dict(t=0.7, k=100, p=0.7003)):
        check(mf, x, noise, **kw)


def test_equal_keys_take_the_lowest_index(mf):
    x = torch.zeros(2, 5000, device="cuda")
    noise = torch.zeros(2, 5000, device="cuda")
    noise[1] = -math.inf
    noise[1, 4000:] = math.nan
    assert run(mf, x, noise)[0] == [0, 0]
    noise[0, 1234] = noise[0, 4321] = 1.0
    assert run(mf, x, noise)[0] == [1234, 0]


def test_strides_and_odd_addresses(mf):
    for dtype in DT:
        big = torch.randn(5, 1013, device="cuda").to(dtype)
        x, noise = big[:, 5:1006], gumbel(5, 1003)[:, 1:1002]
        assert run(mf, x, noise, k=50) == run(mf, x.contiguous(), noise.contiguous(), k=50)


def test_frequencies(mf):
    """Drawn often enough, tokens come up as softmax says: within 5 standard deviations."""
    n, v = 20000, 12
    row = torch.tensor([0.0, 1.0, -1.0, 2.0, 0.5, -3.0, 1.5, -0.5, 0.2, 0.7, -2.0, 1.1], device="cuda")
    got, _ = run(mf, row.expand(n, v).contiguous(), gumbel(n, v, 2), t=0.8)
    p = torch.softmax(row.double() / 0.8, 0).tolist()
    for i in range(v):
        assert abs(got.count(i) - n * p[i]) <= 5 * math.sqrt(n * p[i] * (1 - p[i]))


@pytest.mark.parametrize("dtype", DT)
def test_largest_vocabulary(mf, dtype):
    """2^20 entries: slices that do not fit shared memory, settings that take every path."""
    v = 1 << 20
    g = torch.Generator("cuda").manual_seed(21)
    x = (torch.randn(5, v, device="cuda", generator=g) * 3).to(dtype)
    check(mf, x, gumbel(5, v), t=[1.0, 0.7, 0.0, 1.0, 1.0], k=[0, 40, 3, 60000, 0], p=[1.0, 0.9003, 0.5, 1.0, 0.3003], mp=[0.0, 0.0, 0.0, 0.0, 0.01])


def test_in_a_graph(mf):
    """Captured after another kernel, replayed with other logits and settings."""
    x, noise = torch.randn(4, 5003, device="cuda") * 2, gumbel(4, 5003)
    base, token = x.clone(), torch.empty(4, dtype=torch.int32, device="cuda")
    k = torch.tensor([0, 50, 7, 1000], dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        def body():
            torch.mul(base, 1.5, out=x)
            mf.mf_sample(x, noise, token, top_k=k)
        body()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            body()
        for seed in range(3):
            base.copy_(torch.randn(4, 5003, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)))
            k.copy_(torch.tensor([seed, 50, 7, 1000]))
            g.replay()
            s.synchronize()
            assert token.tolist() == run(mf, base * 1.5, noise, k=k.tolist())[0]


def test_same_every_time(mf):
    x, noise = (torch.randn(64, 50001, device="cuda") * 2).bfloat16(), gumbel(64, 50001)
    a = run(mf, x, noise, t=0.9, k=0, p=0.95)
    for _ in range(5):
        assert run(mf, x, noise, t=0.9, k=0, p=0.95) == a


def test_refusals(mf):
    x, noise, token = torch.zeros(2, 10, device="cuda"), torch.zeros(2, 10, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for a in ((x.double(), noise, token), (x, noise[:, :9], token), (x[:, ::2], noise[:, ::2], token)):
        with pytest.raises(mf.MFError):
            mf.mf_sample(*a)
    ok = dict(logits=x.data_ptr(), noise=noise.data_ptr(), token=token.data_ptr(), logits_stride=10, noise_stride=10, n_rows=2,
              vocab=10, dtype=mf.MF_F32)
    for bad in (dict(logits=None), dict(noise=None), dict(token=None), dict(logits=x.data_ptr() + 2), dict(noise=noise.data_ptr() + 1),
                dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(n_rows=-1), dict(dtype=8), dict(logits_stride=9), dict(noise_stride=9)):
        with pytest.raises(mf.MFError) as e:
            mf._check(mf._lib.mf_sample(mf._SampleArgs(**{**ok, **bad}), None), "mf_sample")
        assert e.value.status == mf.MF_E_INVAL
    mf._check(mf._lib.mf_sample(mf._SampleArgs(**{**ok, "n_rows": 0, "token": None}), None), "mf_sample")


@pytest.mark.parametrize("v", [5003, 131072])
def test_lists_of_all_lengths(mf, v):
    """Entries that are sorted: from a few to as many as the list holds and more."""
    ks = [60, 130, 250, 255, 256, 257, 300, 450, 511, 513, 700, 1400, 2100, 3500, 4090, 4097]
    g = torch.Generator("cuda").manual_seed(v + 7)
    x = torch.randn(len(ks), v, device="cuda", generator=g) * 3
    check(mf, x, gumbel(len(ks), v, v), k=ks)
    check(mf, x, gumbel(len(ks), v, v + 1), k=ks, p=0.9003, t=1.3)


@pytest.mark.parametrize("v", [1000, 50001])
@pytest.mark.parametrize("spread", [0.02, 1.0, 4.0, 20.0])
def test_top_p_of_many(mf, v, spread):
    """From rows where nearly all entries count to rows where most are too small to: p in the middle of an entry's mass.

    Half an entry's share is 1e-5 and more of the total for v = 50001 with p to 0.99, sums and p err by some 1e-7."""
    g = torch.Generator("cuda").manual_seed(v)
    x = torch.randn(1, v, device="cuda", generator=g) * spread
    w = torch.softmax(x[0].double(), 0).sort(descending=True).values
    upto = w.cumsum(0)
    ps = []
    for share in (0.1, 0.5, 0.9, 0.95, 0.99):
        j = int((upto < share).sum())
        p = float(upto[j] - w[j] / 2)
        if w[j] > 4e-6 and p not in ps:
            ps.append(p)
    assert ps
    for mp in (None, [1e-4] * len(ps)):
        check(mf, x.expand(len(ps), v).contiguous(), gumbel(len(ps), v, 3), p=ps, mp=mp)


def test_min_p_close_to_its_entries(mf):
    """Entries whose w is off min_p by 1.5e-6 of it, ten times what an exponential errs by: half are in."""
    v = 3001
    x = torch.full((2, v), math.log(0.5), device="cuda", dtype=torch.float64)
    x[:, ::2] += 1.5e-6
    x[:, 1::2] -= 1.5e-6
    x[:, 1500] = 0.0
    x[1] += 8.0 - x[1].max()  # (coarser logits: 8 + z in steps of 2^-21, the halves stay apart)
    check(mf, x.float(), gumbel(2, v, 11), mp=[0.5, 0.5])


def test_noise_without_bounds(mf):
    """Noise of -inf and NaN rules entries out, one of +inf decides."""
    n, v = 4, 40000
    g = torch.Generator("cuda").manual_seed(31)
    x = torch.randn(n, v, device="cuda", generator=g) * 2
    noise = gumbel(n, v, 17)
    noise[0, torch.rand(v, device="cuda", generator=g) < 0.9] = -math.inf
    noise[1, ::2] = math.nan
    best = int(x[2].argmax())
    noise[2, best] = math.inf
    noise[3, :] = -math.inf
    noise[3, int(x[3].argmax())] = 0.5
    for kw in (dict(), dict(k=5000), dict(k=100), dict(p=0.9003), dict(mp=0.01), dict(p=0.95007, mp=0.003)):
        check(mf, x, noise, **kw)


@pytest.mark.parametrize("v", [4099, 50001])
def test_top_p_is_cut_at_every_border(mf, v):
    """p in steps of one ulp across the masses down to every fourth bin of 1/64 in z: the kept mass is p of the total each
    time, less than an entry too much, and the same again.  (Masses in fp32 err by less than 1e-5 of the total.)"""
    g = torch.Generator("cuda").manual_seed(v + 3)
    x = torch.randn(v, device="cuda", generator=g) * 2
    z = x.double() - x.double().max()
    w, total = z.exp(), z.exp().sum()
    upto = torch.zeros(2049, dtype=torch.float64, device="cuda").index_add_(0, (z * -64).round().clamp(max=2047).long() + 1, w).cumsum(0) / total
    at = upto[::4]
    at = at[(at > 0.03) & (at < 0.97)].float().unique()
    p = (at.view(torch.int32)[:, None] + torch.arange(-24, 25, device="cuda", dtype=torch.int32)).view(-1).view(torch.float32)
    noise = torch.zeros(v, device="cuda")
    noise[x.argmax()] = 100.0
    falling = w.sort(descending=True).values
    before = falling.cumsum(0) - falling
    for q in p.split(512):
        n = len(q)
        rows, token, lp = x.expand(n, v).contiguous(), torch.empty(2, n, dtype=torch.int32, device="cuda"), torch.empty(2, n, device="cuda")
        for i in range(2):
            mf.mf_sample(rows, noise.expand(n, v).contiguous(), token[i], lp[i], top_p=q)
        assert torch.equal(lp[0], lp[1]) and (token == x.argmax()).all()
        held, want = (-lp[0].double()).exp(), q.double() * total
        entry = falling[(torch.searchsorted(before, want) - 2).clamp(min=0)]
        assert (held >= want - 1e-5 * total).all() and (held <= want + 2 * entry + 1e-5 * total).all(), ((held - want) / total).abs().max()


def test_top_p_among_the_first_is_a_prefix(mf):
    """Under top-k too, p in steps of one ulp: the last kept entry (its noise is the largest) and the kept mass agree."""
    v, k = 5003, 2000
    g = torch.Generator("cuda").manual_seed(77)
    x = torch.randn(v, device="cuda", generator=g)
    order = x.argsort(descending=True)
    noise = torch.full((v,), -1e4, device="cuda")
    noise[order] = torch.arange(v, device="cuda").float() * 16  # later entries win whatever their z
    w = (x.double() - x.double().max()).exp()[order][:k]
    upto = w.cumsum(0)
    for i in range(100, 1900, 100):
        p = ((upto[i] / upto[-1]).float().view(torch.int32) + torch.arange(-16, 17, device="cuda", dtype=torch.int32)).view(torch.float32)
        n = len(p)
        token, lp = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
        mf.mf_sample(x.expand(n, v).contiguous(), noise.expand(n, v).contiguous(), token, lp, top_p=p,
                     top_k=torch.full((n,), k, dtype=torch.int32, device="cuda"))
        rank = torch.argsort(order)[token.long()]
        # a sum in fp32 may move the border by an entry or two, what is kept ends there all the same
        assert ((rank - i).abs() <= 2).all(), rank
        held = ((x[token.long()].double() - x.double().max()) - lp.double()).exp()
        assert ((held - upto[rank]).abs() <= 2e-6 * upto[-1]).all(), (rank, (held - upto[rank]) / upto[-1])


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("v", [1 << 18, 1 << 19, 1 << 20])
def test_top_p_beside_large_groups_of_equal_logits(mf, dtype, v):
    """Two large groups of equal logits, one above the border and one below, whose masses a fixed number of bits would round the same
    way entry by entry; the border falls among a few thousand smaller ones.  The noise is such that the last kept one wins.
    Sums of fp32 numbers: 30 roundings of 2^-24 of the total and exponentials off by 2^-22 move the border by at
    most 3e-6 of the total."""
    g = torch.Generator("cuda").manual_seed(v)
    perm = torch.randperm(v, device="cuda", generator=g)
    n_top, n_mid = int(0.4 * v), 3000
    mid = perm[n_top:n_top + n_mid].sort().values  # in the order of their index
    x = torch.full((v,), -1.5, device="cuda")
    noise = torch.full((v,), -100.0, device="cuda")
    noise[mid] = torch.arange(n_mid, device="cuda") * 0.25
    unit = 2.0 ** 34 / v  # of a mass rounded to whole units in slices of an eighth of the row, 2^31 units together
    worst = 0.0
    values = (torch.arange(1, 127, device="cuda") / -16384.0).to(dtype).double()  # of one 1/128 below the largest
    off = (values.exp() * unit).round() - values.exp() * unit
    low = (-1.5 + torch.arange(0, 64, device="cuda") / 4096.0).to(dtype).double()
    place = low + ((low * -64).round() / 64)
    off_low = (place.exp() * unit).round() - place.exp() * unit
    for sign in (1, -1):
        a, b = values[(off * sign).argmax()], low[(off_low * -sign).argmax()]
        y = x.clone().double()
        y[:] = b
        y[perm[:n_top]] = a
        y[mid] = -1.0
        y[perm[-1]] = 0.0
        y = y.to(dtype)
        e = y.double().exp()
        total, above = e.sum(), e[y.double() > -1.0].sum()
        p = [float((above + (j + 0.5) * math.exp(-1.0)) / total) for j in (300, 1200, 1500, 2700)]
        p = torch.tensor(p, dtype=torch.float32, device="cuda")
        want = torch.ceil((p.double() * total - above) / math.exp(-1.0)) - 1  # rank of the last kept one
        n = len(p)
        token = torch.empty(n, dtype=torch.int32, device="cuda")
        mf.mf_sample(y.expand(n, v).contiguous(), noise.expand(n, v).contiguous(), token, None, top_p=p)
        rank = torch.searchsorted(mid, token.long())
        assert torch.equal(mid[rank.clamp(max=n_mid - 1)], token.long())
        worst = max(worst, float((rank - want).abs().max()))
    assert worst <= 1 + 3e-6 * float(total) / math.exp(-1.0), worst


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("v", [7, 4096, 5003, 50001])
def test_ends_of_the_temperature(mf, dtype, v):
    """From the smallest number above 0 to infinity, with forbidden entries, by temperature alone and with cuts."""
    ts = [math.inf, 3e38, 1e38, 1e30, 1e-30, 2.0 ** -120, 1e-39, 1e-45]
    ts = [torch.tensor(t, dtype=torch.float32).item() for t in ts]
    n = len(ts)
    g = torch.Generator("cuda").manual_seed(v + 5)
    x = (torch.randn(n, v, device="cuda", generator=g) * 3).to(dtype)
    x[:, 1::3] = -math.inf
    x[:, 5] = x[:, 0] = x.max(-1).values  # two of the largest at least: noise decides
    left = int((x[0] > -math.inf).sum())
    half = (left // 2 + 0.5) / left
    for kw in (dict(), dict(mp=[0.0] * n), dict(k=[left - 1] * n), dict(k=[max(1, left // 2)] * n), dict(p=[half] * n), dict(mp=[0.5003] * n),
               dict(k=[left // 2 + 2] * n, p=[0.75] * n) if left > 8 else dict()):
        check(mf, x, gumbel(n, v, v), t=ts, **kw)
    x[:, 2] = torch.finfo(dtype).min
    check(mf, x[:, 2:], gumbel(n, v - 2, v), t=ts)
    check(mf, x[:, 2:], gumbel(n, v - 2, v), t=ts, mp=[0.0] * n)


@pytest.mark.parametrize("kw", [dict(), dict(mp=[0.0] * 8), dict(k=[3000] * 8), dict(p=[0.5] * 8)])
def test_infinite_logits_at_the_ends_of_the_temperature(mf, kw):
    """Entries of +inf share the row whatever the temperature."""
    ts = [torch.tensor(t, dtype=torch.float32).item() for t in (math.inf, 3e38, 1.0, 1e-30, 1e-39, 1e-45, 0.0, 5.0)]
    x = torch.randn(8, 4099, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    x[:, ::7] = -math.inf
    x[:, 100::1000] = math.inf
    noise = gumbel(8, 4099, 4)
    got, lp = run(mf, x, noise, t=ts, **kw)
    for r, t in enumerate(ts):
        kept = [100, 1100, 2100, 3100][:1 if t == 0 else 2 if "p" in kw else 4]
        assert got[r] == max(kept, key=lambda i: (noise[r, i].item(), -i))
        assert abs(lp[r] + math.log(len(kept))) <= 2.0 ** -20


@pytest.mark.parametrize("kw", [dict(), dict(mp=[0.0] * 64), dict(k=[20000] * 64)])
def test_large_z_and_noise_that_cancel(mf, kw):
    """z + noise of a far entry comes near that of the largest although both are near 1000: what the products of z err by then is
    a part of 1000, not of their sum."""
    import numpy as np
    n, v, t = 64, 50001, np.float32(1.1)
    rng, far = np.random.default_rng(3), []
    while len(far) < n:  # entries whose z as a product is an ulp (2^-14) above the quotient
        x = np.float32(-rng.uniform(600, 700))
        if np.float32(x * (np.float32(1) / t)) > np.float32(x / t):
            far.append(x)
    x = torch.full((n, v), -1000.0, device="cuda")
    noise = torch.full((n, v), -100.0, device="cuda")
    x[:, 4000], noise[:, 4000] = 0.0, 4.5e-5
    for r, f in enumerate(far):
        x[r, 77] = float(f)
        noise[r, 77] = -float(np.float32(f / t))  # their sum is within half an ulp, 3.1e-5, of 0
        assert float(f) / float(t) - float(np.float32(f / t)) < 3.2e-5
    assert run(mf, x, noise, t=float(t), **kw)[0] == [4000] * n


def test_copies_that_do_not_arrive(mf):
    """Logits that are not there within the wait's limit of a second are read without their copies: the same tokens."""
    import time
    n, v = 5, 50001
    g = torch.Generator("cuda").manual_seed(41)
    t, p, k = [1.0, 0.0, 0.8, 1.0, 1.3], [0.9003, 1.0, 0.95, 1.0, 0.5], [0, 0, 50, 5000, 0]
    with pytest.raises(mf.MFError):
        mf.mf_sample_test_hold(2)
    for dtype in DT:
        x, noise = (torch.randn(n, v, device="cuda", generator=g) * 3).to(dtype), gumbel(n, v, 6)
        x[4] = -math.inf
        got, took = [], []
        for hold in range(2):
            mf.mf_sample_test_hold(hold)
            try:
                t0 = time.perf_counter()
                got.append(run(mf, x, noise, t=t, k=k, p=p))
                took.append(time.perf_counter() - t0)
            finally:
                mf.mf_sample_test_hold(0)
        assert took[0] < 0.5 and 0.9 < took[1] < 10, took
        (token, lp), (held, held_lp) = got
        # sums of the same numbers in another order: 2^6 additions in a thread and ten joins, each errs by 2^-24
        assert token == held and all(a == b or abs(a - b) <= 2.0 ** -17 for a, b in zip(lp, held_lp))
        assert token[4] == -1 and token[0] >= 0


def test_tensors_that_do_not_fit_are_refused(mf):
    """Other types, strides and lengths than the rows' (which would be read as what they are not, or past their end)."""
    n, v = 4, 50
    x, noise = torch.randn(n, v, device="cuda"), gumbel(n, v)
    f, i = torch.ones(n, device="cuda"), torch.full((n,), 20, dtype=torch.int32, device="cuda")
    ok = dict(logits=x, noise=noise, token=torch.full((n,), -7, dtype=torch.int32, device="cuda"), logprob=torch.empty(n, device="cuda"),
              temperature=f, top_k=i, top_p=f * 0.9, min_p=f * 0)
    bad = [dict(noise=noise.half()), dict(noise=noise.double()), dict(noise=noise[0]), dict(noise=noise.cpu()), dict(logits=x.cpu()),
           dict(logits=x.int()), dict(logits=x[0])]
    for name in ("token", "top_k"):
        t = ok[name]
        bad += [{name: y} for y in (t.long(), t.float(), t.short(), t[:n - 1], t.repeat_interleave(2)[::2], t[:1].expand(n), t.cpu())]
    for name in ("logprob", "temperature", "top_p", "min_p"):
        t = ok[name]
        bad += [{name: y} for y in (t.double(), t.half(), t.int(), t[:n - 1], t.repeat_interleave(2)[::2], t[:1].expand(n), t.cpu())]
    for kw in bad:
        with pytest.raises(mf.MFError) as e:
            mf.mf_sample(**{**ok, **kw})
        assert e.value.status == mf.MF_E_INVAL
    torch.cuda.synchronize()
    assert (ok["token"] == -7).all()
    mf.mf_sample(**ok)
    want = ok["token"].tolist()
    # longer ones, columns, and pinned settings serve
    more = {k: torch.cat((t, t)) for k, t in ok.items() if t.dim() == 1}
    mf.mf_sample(x, noise, **more)
    column = torch.empty(n, 1, dtype=torch.int32, device="cuda")
    mf.mf_sample(**{**ok, "token": column, "temperature": f.cpu().pin_memory()})
    mf.mf_sample(**{**ok, "logits": x[:0], "noise": noise[:0]})
    assert more["token"][:n].tolist() == column.view(-1).tolist() == want and (more["token"][n:] == torch.tensor(want, device="cuda")).logical_or(
        more["token"][n:] == -7).all()
