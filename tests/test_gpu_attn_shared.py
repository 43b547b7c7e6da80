"""Attention of sequences that share their first lines against the plain form in 64 bits."""
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


ALL_READ_ALONE = 128e6  # bytes that the tables can hold, up to which every sequence is read by itself


def widen(c):
    """Room in the page tables for so many more lines that the shared ones are read for the group."""
    have, line = c.pages.shape[1], len(c.len) * c.hkv * c.d * 4
    want = max(have, int(ALL_READ_ALONE / (line * c.page)) + 2)
    c.pages = torch.nn.functional.pad(c.pages, (0, want - have)).contiguous()


def share(c, first, lens, copies=False, wide=True):
    """Let groups of the case's sequences begin alike: sequences name the pages of their group's first one (whole pages), or hold
    copies; what is left of a page is copied.  The pages that are no longer named hold NaN."""
    gone = set()
    if wide:
        widen(c)
    for a, b, n in zip(first, first[1:], lens):
        whole = 0 if copies else n // c.page
        for s in range(a + 1, b):
            (pg0, ln0), (pg, ln) = c.lines[a], c.lines[s]
            gone.update(c.pages[s, :whole].tolist())
            c.pages[s, :whole] = c.pages[a, :whole]
            pg = pg.clone()
            pg[:whole * c.page] = pg0[:whole * c.page]
            for x in (c.k, c.v):
                x[pg[:n], ln[:n]] = x[pg0[:n], ln0[:n]]
            c.lines[s] = (pg, ln)
    for p in gone - {int(p) for pg, _ in c.lines for p in pg.unique()}:
        c.k[p] = c.v[p] = math.nan
    i32 = dict(dtype=torch.int32, device="cuda")
    return torch.tensor(first, **i32), torch.tensor(lens, **i32)


def check(mf, c, first, lens, causal=True, scale=None, lse=True, copies=False, status=0, stream=None, q_start=True, lens_given=None):
    scale = 1 / math.sqrt(c.d) if scale is None else scale
    pages = c.pages.shape[1]
    f, n = share(c, first, lens, copies)
    if lens_given is not None:
        n = torch.tensor(lens_given, dtype=torch.int32, device="cuda")
    at = c.attn(mf)
    try:
        mf.mf_attn_share(at, max(1, len(lens)))
        out = torch.full((c.tokens, c.hq, c.d), 7.0, dtype=c.q.dtype, device="cuda")
        le = torch.full((c.tokens, c.hq), 7.0, device="cuda") if lse else None
        want, wl, tol, ltol = ref.attention64(c, scale, 0, causal)
        wide = c.pages
        for c.pages in (wide[:, :pages].contiguous(), wide):  # few lines in the tables: each sequence by itself
            out.fill_(7.0)
            step = c.step(mf) if q_start else c.step(mf, q_start=None)
            for _ in range(2):  # a second call on the same handle finds the workspace as the first left it
                mf.mf_attn_forward_shared(at, mf.kv_cache(c.k, c.v), step, mf.shared(f, n), c.q, out, le, scale, causal=causal, stream=stream)
            assert mf.mf_attn_check(at) == status
            far = (out.double() - want).abs() - tol
            assert not out.isnan().any() and far.max() <= 0, (far.max().item(), (far > 0).sum().item())
            if lse:
                assert torch.equal(le.isinf(), wl.isinf())
                assert ((le.double() - wl).abs() - ltol).nan_to_num(-1).max() <= 0
    finally:
        mf.mf_attn_destroy(at)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 1), (6, 2), (32, 2)])
def test_decode(mf, dtype, d, hq, hkv):
    """One token a sequence: groups of two, three and one, a sequence of no group, prefixes that end inside a page."""
    check(mf, ref.Case([1] * 7, [340, 333, 500, 130, 200, 257, 64], hq, hkv, d, dtype), [0, 2, 5, 6], [333, 100, 250])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 1), (5, 1), (32, 2)])
def test_chunks(mf, dtype, d, hq, hkv):
    """Several tokens a sequence, some sequences with one or none, the group's rows in several tiles."""
    check(mf, ref.Case([5, 1, 0, 130, 33, 64, 1], [300, 304, 290, 400, 200, 229, 190], hq, hkv, d, dtype), [0, 4, 7], [288, 190])


@pytest.mark.parametrize("page,heads_first", [(64, False), (16, True), (24, False), (5, False), (1, False), (256, True)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_pages(mf, d, page, heads_first):
    for new, ctx in (([1] * 5, [1000, 800, 900, 1001, 790]), ([40, 9, 200, 1, 3], [1000, 800, 900, 1001, 790])):
        check(mf, ref.Case(new, ctx, 8, 2, d, page=page, heads_first=heads_first, row_pad=8), [0, 5], [790])


@pytest.mark.parametrize("n,prefix,own", [(2, 4000, 0), (16, 3000, 3), (40, 2049, 100), (3, 128, 2000), (64, 130, 1)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_one_group(mf, n, prefix, own, d):
    """Long and short prefixes, much and little of a sequence's own: work cut between many blocks, or whole in one."""
    c = ref.Case([1] * n, [prefix + (own * i) // n for i in range(n)], 8, 2, d, page=64)
    check(mf, c, [0, n], [prefix])


@pytest.mark.parametrize("d,hq,hkv,new", [(64, 16, 2, [8, 7, 6, 1, 8]), (128, 16, 1, [3, 4, 2, 3, 4]), (128, 8, 4, [20, 33, 17, 40, 1]),
                                          (256, 16, 2, [9, 16, 31, 4, 2]), (256, 5, 1, [12, 40, 9, 50, 33])])
def test_rows_between(mf, d, hq, hkv, new):
    """More rows a sequence than the kernel of few rows holds, fewer than fill tiles of their own."""
    check(mf, ref.Case(new, [600, 580, 700, 577, 1300], hq, hkv, d, page=16), [0, 3, 5], [576, 570])
    check(mf, ref.Case(new, [600, 580, 700, 577, 1300], hq, hkv, d, "f16", page=7), [0, 5], [577], causal=False)


def test_many_tokens(mf):
    """Prompts behind a prefix: tiles of the group that hold several sequences' tokens."""
    check(mf, ref.Case([700, 3, 511, 1, 64, 900], [1030, 1100, 1025, 1024, 1500, 1024], 16, 4, 128), [0, 6], [1024])
    check(mf, ref.Case([300, 301, 302, 303], [600, 500, 700, 800], 16, 4, 256, "f16", page=24), [0, 2, 4], [480, 700])


@pytest.mark.parametrize("n,groups", [(300, 100), (700, 7), (1100, 1100)])
def test_many_sequences(mf, n, groups):
    per = n // groups
    first = [per * i for i in range(groups)] + [n]
    lens = [16 * (1 + i % 7) + i % 5 for i in range(groups)]
    of = [min(i // per, groups - 1) for i in range(n)]
    check(mf, ref.Case([1 + (i % 3 == 0) for i in range(n)], [lens[of[i]] + (i * 37) % 50 for i in range(n)], 4, 2, 64, "f16"), first, lens)


@pytest.mark.parametrize("n", [152, 153, 320])
@pytest.mark.parametrize("d,hq", [(64, 16), (128, 16), (256, 6)])
def test_joins_of_many_blocks(mf, n, d, hq):
    """Two kv heads: as many blocks of the join as two an SM, and more; heads of 256, whose columns then take two rounds."""
    check(mf, ref.Case([1] * n, [500 + (i * 29) % 70 for i in range(n)], hq, 2, d), [0, n // 2, n], [500, 495])


@pytest.mark.parametrize("first,lens", [([0, 0], [0]), ([0, 4], [0]), ([0, 4], [15]), ([0, 4], [16]), ([1, 3], [48]), ([0, 1, 1, 2, 4], [30, 7, 0, 33]),
                                        ([4, 4], [100]), ([0], [])])
def test_groups_of_little(mf, first, lens):
    """No groups, groups of one or no sequence, no line or less than a page in common, sequences beside the groups."""
    check(mf, ref.Case([1, 2, 1, 30], [50, 60, 70, 80], 8, 2, 128), first, lens)


def test_no_lse_no_q_start_and_copies(mf):
    check(mf, ref.Case([1] * 5, [210, 200, 200, 264, 203], 8, 2, 128), [0, 5], [200], lse=False, q_start=False)
    check(mf, ref.Case([1, 3, 1, 9], [210, 200, 200, 264], 8, 2, 128), [0, 4], [200], copies=True)


def test_not_causal(mf):
    for new in ([1, 1, 1], [90, 4, 1]):
        check(mf, ref.Case(new, [100, 90, 300], 4, 2, 128), [0, 3], [90], causal=False)


@pytest.mark.parametrize("new,total", [([1, 1, 1], [0, 5, 40]), ([20, 3, 200], [0, 5, 150])])
def test_rows_that_see_nothing(mf, new, total):
    """Sequences without lines, and tokens whose line would lie before the first, beside a group: zeros and -inf."""
    c = ref.Case(new, [t - n for t, n in zip(total, new)], 8, 2, 128, page=8)
    check(mf, c, [0, 3], [0], status=0 if all(t >= n for t, n in zip(total, new)) else mf.MF_E_INVAL)


@pytest.mark.parametrize("given,first,real", [([300], [0, 3], [100]), ([-5], [0, 3], [0]), ([2 ** 31 - 1], [0, 3], [100])])
def test_lengths_out_of_range(mf, given, first, real):
    """A length that the shortest sequence does not have is taken as what it has; the check says so."""
    check(mf, ref.Case([1, 40, 1], [100, 120, 300], 8, 2, 64), first, real, lens_given=given, status=mf.MF_E_INVAL)


@pytest.mark.parametrize("first", [[2, 0], [-3, 2], [0, 9], [1, 3, 2], [5, 7], [0, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1]])
def test_groups_out_of_range(mf, first):
    """Bounds that fall or lie outside the step are taken as the nearest valid ones."""
    c = ref.Case([1, 2, 1], [100, 100, 100], 8, 2, 64)
    share(c, [0, 3], [100])  # whatever group it is taken for, its sequences begin alike
    at = c.attn(mf)
    mf.mf_attn_share(at, 4)
    f = torch.tensor(first, dtype=torch.int32, device="cuda")
    out = torch.empty(c.tokens, 8, 64, dtype=c.q.dtype, device="cuda")
    mf.mf_attn_forward_shared(at, mf.kv_cache(c.k, c.v), c.step(mf), mf.shared(f, torch.full((len(first) - 1,), 96, dtype=torch.int32, device="cuda")),
                              c.q, out, scale=0.1)
    assert mf.mf_attn_check(at) == mf.MF_E_INVAL and mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)
    want, _, tol, _ = ref.attention64(c, 0.1)
    assert ((out.double() - want).abs() <= tol).all()


def test_large_and_rising_scores(mf):
    """Scores of some hundred, the largest in the prefix or in a sequence's own lines, by which the other part weighs nothing."""
    for up in (True, False):
        c = ref.Case([1, 1, 5], [700, 600, 650], 4, 2, 128)
        f, n = share(c, [0, 3], [600])
        for pg, ln in c.lines:
            ramp = torch.linspace(-3, 3, len(pg), device="cuda") * (1 if up else -1)
            c.k[pg, ln] = ramp.to(c.k.dtype)[:, None, None].expand(-1, 2, 128)
        share(c, [0, 3], [600])
        c.q.fill_(0.5)
        check(mf, c, [0, 3], [600], scale=1.0)


def test_nan_in_q(mf):
    c = ref.Case([1, 2, 1], [400, 390, 500], 8, 2, 128)
    f, n = share(c, [0, 3], [390])
    at = c.attn(mf)
    mf.mf_attn_share(at, 1)
    want, _, tol, _ = ref.attention64(c, 0.1)
    c.q[1, 3, 5] = math.nan
    out, lse = torch.empty(4, 8, 128, dtype=c.q.dtype, device="cuda"), torch.empty(4, 8, device="cuda")
    mf.mf_attn_forward_shared(at, mf.kv_cache(c.k, c.v), c.step(mf), mf.shared(f, n), c.q, out, lse, 0.1)
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)
    hit = torch.zeros(4, 8, dtype=torch.bool, device="cuda")
    hit[1, 3] = True
    assert torch.equal(lse.isnan(), hit) and out[hit].isnan().all() and ((out.double() - want).abs() <= tol)[~hit].all()


def test_output_over_q_and_same_bits(mf):
    for new in ([1] * 4, [40, 200, 1, 2]):
        c = ref.Case(new, [1000, 903, 900, 964], 8, 2, 128)
        first = check(mf, c, [0, 4], [900])
        for _ in range(3):
            assert torch.equal(first, check(mf, c, [0, 4], [900]))
        at = c.attn(mf)
        mf.mf_attn_share(at, 3)
        mf.mf_attn_share(at, 1)  # (again, fewer)
        i32 = dict(dtype=torch.int32, device="cuda")
        mf.mf_attn_forward_shared(at, mf.kv_cache(c.k, c.v), c.step(mf), mf.shared(torch.tensor([0, 4], **i32), torch.tensor([900], **i32)),
                                  c.q, c.q, scale=1 / math.sqrt(128))
        mf.mf_attn_destroy(at)
        assert torch.equal(c.q, first)


def test_offsets_beyond_32_bits(mf):
    base = 2 ** 31 // (64 * 2 * 128) + 1
    for new in ([1, 1], [70, 3]):
        check(mf, ref.Case(new, [300, 330], 8, 2, 128, page=64, base_page=base), [0, 2], [300])


def test_tokens_of_no_sequence(mf):
    c = ref.Case([1, 60], [100, 107], 8, 2, 64)
    f, n = share(c, [0, 2], [100])
    want, _, tol, _ = ref.attention64(c, 0.1)
    at = mf.mf_attn_create(mf.AttnShape(8, 2, 64, mf.MF_BF16), 2, c.tokens + 4, 0)
    mf.mf_attn_share(at, 1)
    for before, after in ((0, 4), (2, 2)):
        rows = before + c.tokens + after
        q = torch.cat((c.q[:before], c.q, c.q[:after]))
        out, lse = torch.full((rows, 8, 64), 7.0, dtype=c.q.dtype, device="cuda"), torch.full((rows, 8), 7.0, device="cuda")
        mf.mf_attn_forward_shared(at, mf.kv_cache(c.k, c.v), mf.step(c.q_start + before, c.kv_len, c.pages, rows, c.max_q), mf.shared(f, n), q,
                                  out, lse, 0.1)
        assert mf.mf_attn_check(at) == mf.MF_E_INVAL
        mine = slice(before, before + c.tokens)
        assert ((out[mine].double() - want).abs() <= tol).all()
        for x in (out, lse):
            assert (x[:before] == 7).all() and (x[before + c.tokens:] == 7).all()
    mf.mf_attn_destroy(at)


def test_beside_plain_calls_in_a_graph(mf):
    """Append, shared and plain attention of one handle captured together on a stream of the caller's, replayed with other lengths of
    prefix and sequences."""
    c = ref.Case([1, 1, 2], [300, 400, 280], 8, 2, 128)
    f, n = share(c, [0, 3], [280])
    at, cache, step = c.attn(mf), mf.kv_cache(c.k, c.v), c.step(mf)
    mf.mf_attn_share(at, 2)
    outs = [torch.empty(4, 8, 128, dtype=c.q.dtype, device="cuda") for _ in range(2)]
    noise = torch.randn_like(c.new_k)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def body():
        c.new_k.add_(noise)
        mf.mf_kv_append(at, cache, step, c.new_k, c.new_v)
        mf.mf_attn_forward_shared(at, cache, step, mf.shared(f, n), c.q, outs[0], scale=0.1)
        mf.mf_attn_forward(at, cache, step, c.q, outs[1], scale=0.1)

    with torch.cuda.stream(s):
        body()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            body()
        full = list(c.lines)
        for lens, prefix in (([301, 401, 282], 280), ([290, 290, 282], 200), ([281, 300, 282], 16), ([281, 300, 282], 0)):
            c.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
            n.fill_(prefix)
            g.replay()
            c.len = lens
            c.lines = [(a[:m], b[:m]) for (a, b), m in zip(full, lens)]
            want, _, tol, _ = ref.attention64(c, 0.1)
            s.synchronize()
            for out in outs:
                assert ((out.double() - want).abs() <= tol).all()
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)


def test_refusals(mf):
    c = ref.Case([3, 1], [10, 15], 8, 2, 64)
    f, n = share(c, [0, 2], [10])
    at, cache, step, group = c.attn(mf), mf.kv_cache(c.k, c.v), c.step(mf), mf.shared(f, n)
    out, lse = torch.empty(4, 8, 64, dtype=c.q.dtype, device="cuda"), torch.empty(4, 8, device="cuda")

    def refused(status=mf.MF_E_INVAL, **kw):
        a = {**dict(attn=at, cache=cache, step=step, shared=group, q=c.q, out=out, lse=lse, scale=0.1), **kw}
        with pytest.raises(mf.MFError) as e:
            mf.mf_attn_forward_shared(**a)
        assert e.value.status == status

    refused(mf.MF_E_STATE)
    for bad in (0, -1, (1 << 20) + 1):
        with pytest.raises(mf.MFError):
            mf.mf_attn_share(at, bad)
    mf.mf_attn_share(at, 1)
    refused(shared=mf.shared(torch.cat((f, f[1:])), torch.cat((n, n))))  # more groups than the handle has room for
    refused(scale=math.nan)
    for t in (c.q.float(), c.q[:3], c.q[:, :4], c.q.cpu(), c.q[..., :32]):
        refused(q=t)
    refused(out=out[:3])
    refused(lse=lse[:3])
    refused(lse=lse.half())
    for make in (lambda: mf.shared(f.cpu(), n.cpu()), lambda: mf.shared(f, n.long()), lambda: mf.shared(n, n)):
        with pytest.raises(ValueError):
            make()
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [lambda i: 1, lambda i: 30 if i % 50 == 0 else 1 + (i % 7 == 0), lambda i: int(i % 60 == 1)],
                         ids=["single tokens", "some with many rows", "most without tokens"])
def test_many_sequences_that_share(mf, d, new):
    """More sequences than the plan holds in shared memory, with lines in common: those of few rows, of many, and groups that have few rows
    themselves.  The same bits again, also beside another stream's kernels, which let the plan's blocks begin at different times."""
    n, first, lens = 1100, [0, 3, 400, 1090], [70, 33, 100]
    of = [sum(i >= f for f in first[1:]) for i in range(n)]
    c = ref.Case([new(i) for i in range(n)], [(lens + [0])[of[i]] + (i * 37) % 50 for i in range(n)], 4, 2, d, "f16")
    want = check(mf, c, first, lens)
    at, i32 = c.attn(mf), dict(dtype=torch.int32, device="cuda")
    mf.mf_attn_share(at, 3)
    groups = mf.shared(torch.tensor(first, **i32), torch.tensor(lens, **i32))
    outs = torch.full((40, *want.shape), 7.0, dtype=want.dtype, device="cuda")
    other, x = torch.cuda.Stream(), torch.randn(2048, 2048, device="cuda")
    other.wait_stream(torch.cuda.current_stream())
    for out in outs:
        with torch.cuda.stream(other):
            for _ in range(3):
                x.mul_(0.5)
        mf.mf_attn_forward_shared(at, mf.kv_cache(c.k, c.v), c.step(mf), groups, c.q, out, scale=1 / math.sqrt(d))
    torch.cuda.synchronize()
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)
    assert (outs.view(torch.int16) == want.view(torch.int16)).all()


@pytest.mark.parametrize("long", [False, True])
def test_many_groups_of_several(mf, long):
    """More groups than the plan holds in shared memory, each with lines in common, on the list of few rows and on that of many."""
    n, per = 900, 3
    lens = [16 * (1 + g % 5) + g % 3 for g in range(n // per)]
    c = ref.Case([1 + 40 * (long and i % 90 == 4) for i in range(n)], [lens[i // per] + (i * 37) % 40 for i in range(n)], 4, 2, 64, "f16")
    first = check(mf, c, list(range(0, n + 1, per)), lens)
    assert torch.equal(first, check(mf, c, list(range(0, n + 1, per)), lens))
