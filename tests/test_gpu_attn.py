"""Paged attention and the append with rotation against the plain forms in 64 bits."""
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


def check(mf, c, window=0, causal=True, scale=None, lse=True, q_start=True, stream=None):
    scale = 1 / math.sqrt(c.d) if scale is None else scale
    at = c.attn(mf)
    try:
        out = torch.full((c.tokens, c.hq, c.d), 7.0, dtype=c.q.dtype, device="cuda")
        le = torch.full((c.tokens, c.hq), 7.0, device="cuda") if lse else None
        step = c.step(mf) if q_start else c.step(mf, q_start=None)
        for _ in range(2):  # a second call on the same handle finds the workspace as the first left it
            mf.mf_attn_forward(at, mf.kv_cache(c.k, c.v), step, c.q, out, le, scale, window=window, causal=causal, stream=stream)
        assert mf.mf_attn_check(at) == (0 if all(n >= m for n, m in zip(c.len, c.new)) else mf.MF_E_INVAL)
    finally:
        mf.mf_attn_destroy(at)
    want, wl, tol, ltol = ref.attention64(c, scale, window, causal)
    far = (out.double() - want).abs() - tol
    assert not out.isnan().any() and far.max() <= 0, (far.max().item(), (far > 0).sum().item())
    if lse:
        assert torch.equal(le.isinf(), wl.isinf())
        assert ((le.double() - wl).abs() - ltol).nan_to_num(-1).max() <= 0
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 1), (6, 2), (32, 2)])
def test_decode(mf, dtype, d, hq, hkv):
    """One token a sequence: lengths of one, around a tile's and a page's end, and longer."""
    check(mf, ref.Case([1] * 9, [0, 1, 15, 16, 62, 63, 64, 130, 700], hq, hkv, d, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 1), (5, 1), (32, 2)])
def test_chunks(mf, dtype, d, hq, hkv):
    """Several tokens a sequence, some sequences with one or none."""
    check(mf, ref.Case([5, 1, 0, 130, 33, 64, 1], [0, 200, 9, 100, 31, 129, 0], hq, hkv, d, dtype))


@pytest.mark.parametrize("page,heads_first", [(64, False), (16, True), (24, False), (5, False)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_long_prompts(mf, d, page, heads_first):
    """Blocks that walk many segments: tiles that are copied whole and by lines take turns in the ring."""
    check(mf, ref.Case([1500, 3, 900, 1, 1999, 640], [0, 700, 37, 1300, 0, 2000], 16, 4, d, page=page, heads_first=heads_first))
    check(mf, ref.Case([900, 1999], [300, 0], 16, 4, d, "f16", page=page, heads_first=heads_first), window=200)


@pytest.mark.parametrize("new,ctx", [([1], [0]), ([1], [40000]), ([3], [9000]), ([700], [0]), ([257], [2000]), ([16], [112])])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_one_sequence(mf, new, ctx, d):
    """One sequence: work split over its lines."""
    check(mf, ref.Case(new, ctx, 8, 2, d, page=64))


@pytest.mark.parametrize("page", [1, 7, 24, 256])
@pytest.mark.parametrize("heads_first", [False, True])
def test_pages_and_strides(mf, page, heads_first):
    """Page sizes that end inside a tile, lines by head or by token, q as part of a wider row."""
    for new in ([1, 1, 1], [40, 9, 2]):
        check(mf, ref.Case(new, [300, 5, 77], 8, 2, 128, page=page, heads_first=heads_first, row_pad=8))


@pytest.mark.parametrize("window", [1, 5, 64, 100, 5000])
@pytest.mark.parametrize("d", [64, 256])
def test_window(mf, window, d):
    """Sliding windows: lines before every window hold garbage and are on pages that are no longer there."""
    for new, ctx in (([1, 1, 1], [500, 3, 64]), ([5, 70, 300], [400, 0, 129])):
        c = ref.Case(new, ctx, 8, 2, d)
        for s, n in enumerate(c.len):
            gone = max(0, n - new[s] - window + 1)  # lines that no token of the step sees
            c.k[c.lines[s][0][:gone], c.lines[s][1][:gone]] = math.inf
            c.v[c.lines[s][0][:gone], c.lines[s][1][:gone]] = math.nan
        check(mf, c, window=window)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_not_causal(mf, d):
    """Every token sees the whole sequence; with a window, the lines from its start on."""
    for new, ctx in (([1, 1], [100, 0]), ([90, 4], [100, 0])):
        check(mf, ref.Case(new, ctx, 4, 2, d), causal=False)
        check(mf, ref.Case(new, ctx, 4, 2, d), causal=False, window=33)


@pytest.mark.parametrize("new,total", [([1, 1, 1], [0, 5, 0]), ([20, 3, 200], [0, 5, 150])])
def test_rows_that_see_nothing(mf, new, total):
    """A sequence of no lines, and tokens whose line would lie before the first: zeros and -inf."""
    check(mf, ref.Case(new, [t - n for t, n in zip(total, new)], 8, 2, 128, page=8))


def test_no_lse_and_no_q_start(mf):
    check(mf, ref.Case([1] * 5, [10, 0, 200, 64, 3], 8, 2, 128), lse=False, q_start=False)


@pytest.mark.parametrize("n,new", [(700, 1), (300, 3)])
def test_many_sequences(mf, n, new):
    check(mf, ref.Case([new] * n, [(i * 37) % 90 for i in range(n)], 4, 2, 64, "f16"))


def test_large_scores(mf):
    """Scores of some hundred, whose exponentials overflow unless the maximum is taken off."""
    for new in ([1], [130]):
        c = ref.Case(new, [500], 4, 2, 128)
        c.q.mul_(30)
        check(mf, c, scale=1.0)


def test_rising_scores(mf):
    """The maximum grows from line to line, so that every tile rescales what was summed."""
    for new in ([1], [20], [150]):
        c = ref.Case(new, [1000], 4, 1, 64)
        pg, ln = c.lines[0]
        c.k[pg, ln] = torch.linspace(-3, 3, len(pg), device="cuda").to(c.k.dtype)[:, None, None].expand(-1, 1, 64)
        c.q.fill_(0.5)
        check(mf, c, scale=1.0)


def test_offsets_beyond_32_bits(mf):
    """Pages whose offset passes 2^31 elements."""
    base = 2 ** 31 // (64 * 2 * 128) + 1
    for new in ([1, 1], [70, 3]):
        c = ref.Case(new, [200, 30], 8, 2, 128, page=64, base_page=base)
        check(mf, c)
        append(mf, c, None)


def test_other_stream_and_graph(mf):
    """On a stream of the caller's, captured once and replayed with other lengths."""
    c = ref.Case([1, 1, 1], [500, 20, 0], 8, 2, 128)
    at, cache, step = c.attn(mf), mf.kv_cache(c.k, c.v), c.step(mf)
    out = torch.empty(3, 8, 128, dtype=c.q.dtype, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        mf.mf_attn_forward(at, cache, step, c.q, out, scale=0.1)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            mf.mf_attn_forward(at, cache, step, c.q, out, scale=0.1)
        for lens in ([501, 21, 1], [77, 21, 1], [301, 1, 1]):
            c.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
            c.len = lens
            c.lines = [(a[:n], b[:n]) for (a, b), n in zip(c.lines, (501, 21, 1))]
            view = ref.Case.__new__(ref.Case)
            view.__dict__.update(c.__dict__)
            view.lines = [(a[:n], b[:n]) for (a, b), n in zip(c.lines, lens)]
            g.replay()
            want, _, tol, _ = ref.attention64(view, 0.1)
            s.synchronize()
            assert ((out.double() - want).abs() <= tol).all()
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)


@pytest.mark.parametrize("new", [1, 70])
def test_step_in_a_graph(mf, new):
    """Append and attention captured together after other work, replayed with other lengths and tokens."""
    c = ref.Case([new, new], [300, 20], 8, 2, 128)
    at, cache, step = c.attn(mf), mf.kv_cache(c.k, c.v), c.step(mf)
    out = torch.empty(c.tokens, 8, 128, dtype=c.q.dtype, device="cuda")
    noise = torch.randn_like(c.new_k)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def body():
        c.new_k.add_(noise)  # (another kernel, and a copy, before)
        c.new_v.copy_(noise)
        mf.mf_kv_append(at, cache, step, c.new_k, c.new_v)
        mf.mf_attn_forward(at, cache, step, c.q, out, scale=0.1)

    with torch.cuda.stream(s):
        body()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            body()
        full = list(c.lines)
        for lens in (c.len, [new + 77, new], [new + 300, new + 1]):
            c.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
            g.replay()
            c.len = lens
            c.lines = [(a[:n], b[:n]) for (a, b), n in zip(full, lens)]
            want, _, tol, _ = ref.attention64(c, 0.1)
            s.synchronize()
            for i, (pg, ln) in enumerate(c.lines):
                rows = slice(c.start[i], c.start[i + 1])
                assert torch.equal(c.k[pg[-new:], ln[-new:]], c.new_k[rows]) and torch.equal(c.v[pg[-new:], ln[-new:]], c.new_v[rows])
            assert ((out.double() - want).abs() <= tol).all()
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)


def test_same_bits_every_time(mf):
    for new, ctx in (([1] * 4, [3000, 7, 900, 64]), ([40, 200], [1000, 3])):
        c = ref.Case(new, ctx, 8, 2, 128)
        first = check(mf, c)
        for _ in range(3):
            assert torch.equal(first, check(mf, c))


def test_output_over_q(mf):
    for new, ctx in (([1, 1], [700, 3]), ([90, 3], [700, 3])):
        c = ref.Case(new, ctx, 8, 2, 128)
        want, _, tol, _ = ref.attention64(c, 0.1)
        at = c.attn(mf)
        mf.mf_attn_forward(at, mf.kv_cache(c.k, c.v), c.step(mf), c.q, c.q, scale=0.1)
        assert ((c.q.double() - want).abs() <= tol).all()
        mf.mf_attn_destroy(at)


def test_bad_pages_are_reported(mf):
    """A page outside the pool is never followed; the check says so once."""
    for new in ([1], [40]):
        c = ref.Case(new, [100], 8, 2, 64)
        c.k.nan_to_num_(0), c.v.nan_to_num_(0)
        c.pages[0, 2] = 1 << 30
        c.pages[0, 3] = -5
        at = c.attn(mf)
        out = torch.empty(c.tokens, 8, 64, dtype=c.q.dtype, device="cuda")
        mf.mf_attn_forward(at, mf.kv_cache(c.k, c.v), c.step(mf), c.q, out)
        assert mf.mf_attn_check(at) == mf.MF_E_INVAL and mf.mf_attn_check(at) == 0
        assert out.isfinite().all()
        before = c.k.clone()
        c.kv_len.fill_(40)  # line 39, on page 2
        if new == [1]:
            mf.mf_kv_append(at, mf.kv_cache(c.k, c.v), c.step(mf), c.new_k, c.new_v)
            assert mf.mf_attn_check(at) == mf.MF_E_INVAL and torch.equal(before, c.k)
        mf.mf_attn_destroy(at)


def append(mf, c, rot, interleaved=False, sections=None, in_place=False):
    """Append c's new tokens and compare with the plain form; rot None: no rotation."""
    at, u = c.attn(mf), ref.U[c.dtype]
    rope = cos = sin = None
    line = torch.cat([torch.arange(n - m, n, device="cuda") for n, m in zip(c.len, c.new)])
    if rot:
        half, n_pos = rot // 2, 50000
        ang = torch.rand(n_pos, half, device="cuda", dtype=torch.float64) * 6.3
        tc, ts = ang.cos().float(), ang.sin().float()
        if sections:
            pos = torch.randint(0, n_pos, (len(sections), c.tokens), dtype=torch.int32, device="cuda")
            axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections)).cuda()
            p = pos[axis].t().long()
            pair = torch.arange(half, device="cuda")
            cos, sin = tc[p, pair], ts[p, pair]
        else:
            pos, cos, sin = None, tc[line], ts[line]
        rope = mf.rope(tc, ts, pos, interleaved, sections)
    q, k, v = c.q.clone() if in_place else c.q, c.new_k, c.new_v
    q_out = q if in_place else torch.empty(c.tokens, c.hq, c.d, dtype=q.dtype, device="cuda")
    q0, kc, vc = q.clone(), c.k.clone(), c.v.clone()
    mf.mf_kv_append(at, mf.kv_cache(c.k, c.v), c.step(mf), k, v, q, q_out, rope)
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)
    pg = torch.cat([a[n - m:n] for (a, b), n, m in zip(c.lines, c.len, c.new)])
    ln = torch.cat([b[n - m:n] for (a, b), n, m in zip(c.lines, c.len, c.new)])
    for got, x in ((q_out, q0), (c.k[pg, ln], k)):
        if rot:
            want, size = ref.rotate64(x, cos, sin, interleaved)
            tol = u * want.abs() + 3 * 2.0 ** -24 * size + (2.0 ** -25 if c.dtype == "f16" else 0)  # one rounding, three in fp32
            assert ((got.double() - want).abs() <= tol * 1.001).all()
        else:
            assert torch.equal(got, x)
    assert torch.equal(c.v[pg, ln], v)
    for got, was in ((c.k, kc), (c.v, vc)):  # nothing else is touched
        got[pg, ln] = was[pg, ln]
        assert torch.equal(got.view(torch.int16), was.view(torch.int16))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 16), (128, 128), (128, 48), (256, 64), (256, 256)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append(mf, dtype, d, rot, interleaved):
    append(mf, ref.Case([5, 1, 0, 130, 1], [0, 200, 9, 100, 16], 6, 2, d, dtype, page=24), rot, interleaved)


@pytest.mark.parametrize("sections", [(8, 12, 12), (0, 32), (11, 10, 6, 5)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_axes(mf, sections, interleaved):
    append(mf, ref.Case([7, 300], [0, 5], 4, 4, 128, heads_first=True, row_pad=16), 64, interleaved, sections)


def test_append_copies_without_rotation(mf):
    append(mf, ref.Case([1] * 300, [i % 50 for i in range(300)], 4, 1, 128, page=1), None)


def test_append_in_place(mf):
    append(mf, ref.Case([9, 1], [3, 64], 8, 2, 128), 128, in_place=True)


def test_append_positions_out_of_range(mf):
    c = ref.Case([2], [10], 4, 2, 64)
    at = c.attn(mf)
    cos, sin = torch.ones(8, 32, device="cuda"), torch.zeros(8, 32, device="cuda")
    pos = torch.tensor([3, 8], dtype=torch.int32, device="cuda")
    mf.mf_kv_append(at, mf.kv_cache(c.k, c.v), c.step(mf), c.new_k, c.new_v, rope=mf.rope(cos, sin, pos))
    assert mf.mf_attn_check(at) == mf.MF_E_INVAL
    pg, ln = c.lines[0]
    assert torch.equal(c.k[pg[10:], ln[10:]], c.new_k)
    mf.mf_attn_destroy(at)


def test_refusals(mf):
    c = ref.Case([3, 1], [10, 5], 8, 2, 64)
    at, cache, step = c.attn(mf), mf.kv_cache(c.k, c.v), c.step(mf)
    out = torch.empty(c.tokens, 8, 64, dtype=c.q.dtype, device="cuda")

    def refused(call, *a, **kw):
        with pytest.raises(mf.MFError) as e:
            call(*a, **kw)
        assert e.value.status == mf.MF_E_INVAL

    def changed(make, **kw):
        s = make()
        for k, v in kw.items():
            setattr(s, k, v)
        return s

    def fwd(cache=cache, step=step, **kw):
        refused(mf.mf_attn_forward, at, cache, step, kw.pop("q", c.q), kw.pop("out", out), **kw)

    for kw in (dict(k=None), dict(v=c.v.data_ptr() + 2), dict(page_stride=9), dict(head_stride=-8), dict(page_size=0),
               dict(n_pages=0)):
        fwd(cache=changed(lambda: mf.kv_cache(c.k, c.v), **kw))
    for kw in (dict(n_seqs=3), dict(n_tokens=5), dict(n_tokens=-1), dict(max_q=0), dict(kv_len=None), dict(pages=None),
               dict(pages_per_seq=0), dict(q_start=None)):
        fwd(step=changed(lambda: c.step(mf), **kw))
    fwd(window=-1)
    fwd(scale=math.inf)
    fwd(q=c.q.transpose(1, 2))
    fwd(q=torch.empty(c.tokens * 8 * 64 + 1, dtype=c.q.dtype, device="cuda")[1:].view(c.tokens, 8, 64))
    fwd(out=torch.empty(c.tokens, 516, dtype=c.q.dtype, device="cuda")[:, :512].unflatten(1, (8, 64)))
    with pytest.raises(mf.MFError):
        mf.mf_attn_forward(None, cache, step, c.q, out)
    cos = torch.ones(64, 32, device="cuda")
    good = mf.rope(cos, cos)
    for kw in (dict(cos=None), dict(n_pos=0), dict(rot_dim=24), dict(rot_dim=80), dict(n_axes=0), dict(n_axes=5),
               dict(n_axes=2)):
        refused(mf.mf_kv_append, at, cache, step, c.new_k, c.new_v, rope=changed(lambda: mf.rope(cos, cos), **kw))
    pos = torch.zeros(2, c.tokens, dtype=torch.int32, device="cuda")
    refused(mf.mf_kv_append, at, cache, step, c.new_k, c.new_v, rope=mf.rope(cos, cos, pos, sections=(16, 15)))
    refused(mf.mf_kv_append, at, cache, step, c.new_k, c.new_v, q=c.q, rope=good)  # q without q_out
    empty = changed(lambda: c.step(mf), n_tokens=0)
    mf.mf_attn_forward(at, cache, empty, c.q, out)  # nothing to do
    mf.mf_kv_append(at, cache, empty, c.new_k, c.new_v)
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)


@pytest.mark.parametrize("window", [2 ** 30 - 1, 2 ** 30, 2 ** 31 - 5, 2 ** 31 - 1])
@pytest.mark.parametrize("new,total", [([1, 1, 4], [0, 5, 1]), ([20, 3, 200], [0, 5, 150])])
@pytest.mark.parametrize("causal", [True, False])
def test_largest_windows(mf, window, new, total, causal):
    """Windows as long as their type allows hide nothing, also from tokens whose line would lie before the first."""
    c = ref.Case(new, [t - n for t, n in zip(total, new)], 8, 2, 128)
    assert torch.equal(check(mf, c, window=window, causal=causal), check(mf, c, causal=causal))


@pytest.mark.parametrize("new,ctx", [([1, 1, 2], [40, 5, 900]), ([1], [5000]), ([90, 3, 200], [40, 5, 900]), ([40], [5000])])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_nan_in_q(mf, new, ctx, d):
    """A token whose q holds NaN: its heads' out and lse are NaN (not the -inf of one that sees nothing), all others what they were."""
    c = ref.Case(new, ctx, 8, 2, d)
    at, cache, step = c.attn(mf), mf.kv_cache(c.k, c.v), c.step(mf)
    want, _, tol, _ = ref.attention64(c, 0.1)
    got = []
    bad = [(0, 3), (c.tokens - 1, 0), (c.tokens // 2, 7)]
    for _ in range(2):
        out, lse = torch.empty(c.tokens, 8, d, dtype=c.q.dtype, device="cuda"), torch.empty(c.tokens, 8, device="cuda")
        mf.mf_attn_forward(at, cache, step, c.q, out, lse, 0.1)
        got.append((out, lse))
        for t, h in bad:
            c.q[t, h, 5] = math.nan
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)
    hit = torch.zeros(c.tokens, 8, dtype=torch.bool, device="cuda")
    for t, h in bad:
        hit[t, h] = True
    (_, lse0), (out1, lse1) = got
    assert lse0.isfinite().all() and torch.equal(lse1.isnan(), hit) and (lse1 - lse0)[~hit].abs().max() < 1e-5
    assert out1[hit].isnan().all() and ((out1.double() - want).abs() <= tol)[~hit].all()


@pytest.mark.parametrize("new", [[1, 3], [60, 70]])
def test_tokens_of_no_sequence_are_reported(mf, new):
    """Tokens before the first sequence's or after the last one's: the check says so after attention as it does after an append; their
    rows stay, the others are right."""
    c = ref.Case(new, [100, 7], 8, 2, 64)
    want, _, tol, _ = ref.attention64(c, 0.1)
    at = mf.mf_attn_create(mf.AttnShape(8, 2, 64, mf.MF_BF16), 2, c.tokens + 4, 0)
    cache = mf.kv_cache(c.k, c.v)
    for before, after in ((0, 4), (2, 0), (2, 2)):
        n = before + c.tokens + after
        q, k, v = (torch.cat((x[:before], x, x[:after])) for x in (c.q, c.new_k, c.new_v))
        out, lse = torch.full((n, 8, 64), 7.0, dtype=c.q.dtype, device="cuda"), torch.full((n, 8), 7.0, device="cuda")
        step = mf.step(c.q_start + before, c.kv_len, c.pages, n, c.max_q)
        mf.mf_attn_forward(at, cache, step, q, out, lse, 0.1)
        assert mf.mf_attn_check(at) == mf.MF_E_INVAL and mf.mf_attn_check(at) == 0
        mine = slice(before, before + c.tokens)
        assert ((out[mine].double() - want).abs() <= tol).all()
        for x in (out, lse):
            assert (x[:before] == 7).all() and (x[before + c.tokens:] == 7).all()
        mf.mf_kv_append(at, mf.kv_cache(c.k.clone(), c.v.clone()), step, k, v)
        assert mf.mf_attn_check(at) == mf.MF_E_INVAL
    mf.mf_attn_destroy(at)


def test_tensors_that_do_not_fit_are_refused(mf):
    """Other types, heads, sizes and lengths than the handle's and the step's, which would be read or written past their end."""
    c = ref.Case([3, 1], [10, 5], 8, 2, 64)
    at, cache, step = c.attn(mf), mf.kv_cache(c.k, c.v), c.step(mf)
    out, lse = torch.empty(4, 8, 64, dtype=c.q.dtype, device="cuda"), torch.empty(4, 8, device="cuda")

    def others(t):
        return (t.float(), t.half(), t[:3], t[:, :-1], t[:, :, :32], t.cpu(), t.contiguous().view(4, t.shape[1] * 2, 32), t[0])

    def refused(call, **kw):
        with pytest.raises(mf.MFError) as e:
            call(**kw)
        assert e.value.status == mf.MF_E_INVAL

    fwd = dict(attn=at, cache=cache, step=step, q=c.q, out=out, lse=lse, scale=0.1)
    for name in ("q", "out"):
        for t in others(fwd[name]):
            refused(mf.mf_attn_forward, **{**fwd, name: t})
    for t in (lse.double(), lse.half(), lse[:3], lse.repeat(1, 2)[:, ::2], lse.t().contiguous().t(), lse.cpu()):
        refused(mf.mf_attn_forward, **{**fwd, "lse": t})
    app = dict(attn=at, cache=cache, step=step, k=c.new_k, v=c.new_v, q=c.q, q_out=out)
    for name in ("k", "v", "q", "q_out"):
        for t in others(app[name]):
            refused(mf.mf_kv_append, **{**app, name: t})
    cos = torch.ones(64, 32, device="cuda")
    for pos, sections in ((torch.zeros(3, dtype=torch.int32, device="cuda"), None), (torch.zeros(2, 3, dtype=torch.int32, device="cuda"), (16, 16)),
                          (torch.zeros(2, 5, dtype=torch.int32, device="cuda"), (16, 16))):
        refused(mf.mf_kv_append, rope=mf.rope(cos, cos, pos, sections=sections), **app)
    for k, v in ((c.k[:, :, :1], c.v[:, :, :1]), (c.k[..., :32], c.v[..., :32]), (c.k.half(), c.v.half())):
        refused(mf.mf_attn_forward, **{**fwd, "cache": mf.kv_cache(k, v)})
        refused(mf.mf_kv_append, **{**app, "cache": mf.kv_cache(k, v)})
    for make in (lambda: mf.kv_cache(c.k.cpu(), c.v.cpu()), lambda: mf.rope(cos.cpu(), cos.cpu()),
                 lambda: mf.step(c.q_start, c.kv_len.cpu(), c.pages, 4, 3)):
        with pytest.raises(ValueError):
            make()
    # more rows than the step has tokens are as good
    want, _, tol, _ = ref.attention64(c, 0.1)
    big = torch.full((9, 8, 64), 7.0, dtype=out.dtype, device="cuda")
    mf.mf_attn_forward(at, cache, step, torch.cat((c.q, c.q)), big, torch.empty(100, device="cuda"), 0.1)
    assert ((big[:4].double() - want).abs() <= tol).all() and (big[4:] == 7).all()
    mf.mf_kv_append(at, cache, step, c.new_k, c.new_v, c.q, big, mf.rope(cos, cos, torch.zeros(9, dtype=torch.int32, device="cuda")))
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)
    refused(mf.mf_attn_forward, **fwd)  # (a handle that is gone)


@pytest.mark.parametrize("hq,hkv", [(4, 1), (1, 1)])
def test_one_head_of_any_head_stride(mf, hq, hkv):
    """The stride between heads of a tensor that has one head means nothing: rows as a transpose of [head][token][dim] leaves them."""
    c = ref.Case([3, 1], [10, 5], hq, hkv, 64)
    turned = [x.transpose(0, 1).contiguous().transpose(0, 1) if x.shape[1] == 1 else x.contiguous() for x in (c.q, c.new_k, c.new_v)]
    assert turned[1].stride() == (64, 256, 1)
    c.q, c.new_k, c.new_v = turned
    check(mf, c)
    append(mf, c, 64)
