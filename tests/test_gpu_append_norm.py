"""The append with norms of q and k against the plain form in 64 bits."""
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


def norm64(x, w, eps, offset):
    if w is None:
        return x.double()
    x = x.double()
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * (w.double() + offset)


def weights(c, f32=False, seed=0, centre=1.0):
    g = torch.Generator("cuda").manual_seed(seed + 5)
    return [(centre + 0.4 * torch.randn(c.d, device="cuda", generator=g)).to(torch.float32 if f32 else c.q.dtype) for _ in range(2)]


def check(mf, c, rot, interleaved=False, sections=None, in_place=False, w=None, eps=1e-6, offset=0.0, with_q=True, stream=None):
    """Tolerance: the sum of squares is off by at most 20 roundings (16 products and sums, 4 over lanes), its root by half of that,
    rsqrt by 2 ulp (4 units), the products with it, with the weight, and the weight's offset by one each: 18 units of 2^-24; the
    rotation adds two of its terms' sum; 24 are allowed for.  Then one rounding to the type (in fp16 half of its smallest step at least)."""
    at, u = c.attn(mf), ref.U[c.dtype]
    qw, kw = weights(c) if w is None else w
    rope = cos = sin = None
    line = torch.cat([torch.arange(n - m, n, device="cuda") for n, m in zip(c.len, c.new)])
    if rot:
        half, n_pos = rot // 2, 50000
        ang = torch.rand(n_pos, half, device="cuda", dtype=torch.float64) * 6.3
        tc, ts = ang.cos().float(), ang.sin().float()
        if sections:
            pos = torch.randint(0, n_pos, (len(sections), c.tokens), dtype=torch.int32, device="cuda")
            axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections)).cuda()
            p, pair = pos[axis].t().long(), torch.arange(half, device="cuda")
            cos, sin = tc[p, pair], ts[p, pair]
        else:
            pos, cos, sin = None, tc[line], ts[line]
        rope = mf.rope(tc, ts, pos, interleaved, sections)
    q, k, v = c.q.clone() if in_place else c.q, c.new_k, c.new_v
    q_out = q if in_place else torch.empty(c.tokens, c.hq, c.d, dtype=q.dtype, device="cuda")
    q0, kc, vc = q.clone(), c.k.clone(), c.v.clone()
    mf.mf_kv_append_norm(at, mf.kv_cache(c.k, c.v), c.step(mf), mf.qk_norm(qw, kw, eps, offset), k, v, q if with_q else None,
                         q_out if with_q else None, rope, stream=stream)
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)
    pg = torch.cat([a[n - m:n] for (a, b), n, m in zip(c.lines, c.len, c.new)])
    ln = torch.cat([b[n - m:n] for (a, b), n, m in zip(c.lines, c.len, c.new)])
    for got, x, weight in ((q_out, q0, qw), (c.k[pg, ln], k, kw))[0 if with_q else 1:]:
        want = size = norm64(x, weight, eps, offset)
        size = size.abs()
        if rot:
            want, size = ref.rotate64(want, cos, sin, interleaved)
        if weight is None and not rot:
            assert torch.equal(got, x)
            continue
        tol = u * want.abs() + 24 * 2.0 ** -24 * size + (2.0 ** -25 if c.dtype == "f16" else 0)
        assert ((got.double() - want).abs() <= tol * 1.01).all()
    assert torch.equal(c.v[pg, ln].view(torch.int16), v.contiguous().view(torch.int16))
    for got, was in ((c.k, kc), (c.v, vc)):  # nothing else is touched
        got[pg, ln] = was[pg, ln]
        assert torch.equal(got.view(torch.int16), was.view(torch.int16))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 16), (128, 128), (128, 48), (256, 64), (256, 256)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append(mf, dtype, d, rot, interleaved):
    check(mf, ref.Case([5, 1, 0, 130, 1], [0, 200, 9, 100, 16], 6, 2, d, dtype, page=24), rot, interleaved, offset=1.0,
          w=[x - 1 for x in weights(ref.Case([1], [0], d=d, dtype=dtype))])


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 5), (40, 8), (64, 4), (96, 32)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_heads(mf, hq, hkv, d):
    """Heads that fill rows of a warp and warps in part."""
    check(mf, ref.Case([1, 7], [3, 0], hq, hkv, d), d)


@pytest.mark.parametrize("sections", [(8, 12, 12), (0, 32), (11, 10, 6, 5)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_axes(mf, sections, interleaved):
    check(mf, ref.Case([7, 300], [0, 5], 4, 4, 128, heads_first=True, row_pad=16), 64, interleaved, sections)


@pytest.mark.parametrize("page", [1, 7, 64])
def test_many_sequences_without_rotation(mf, page):
    check(mf, ref.Case([1] * 300, [i % 50 for i in range(300)], 4, 1, 128, page=page), None)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("which", [(True, False), (False, True), (False, False)])
def test_one_norm_or_none(mf, f32, which):
    c = ref.Case([9, 1], [3, 64], 8, 2, 128)
    w = [x if yes else None for x, yes in zip(weights(c, f32), which)]
    check(mf, c, 128, w=w)
    check(mf, c, None, w=w)


def test_weights_in_32_bits(mf):
    c = ref.Case([40, 3], [0, 9], 8, 2, 64, "f16")
    check(mf, c, 32, True, w=weights(c, True), eps=1e-3, offset=0.5)


def test_in_place_and_without_q(mf):
    check(mf, ref.Case([9, 1], [3, 64], 8, 2, 128), 128, in_place=True)
    check(mf, ref.Case([9, 1], [3, 64], 8, 2, 128), 128, with_q=False)


def test_offsets_beyond_32_bits(mf):
    base = 2 ** 31 // (64 * 2 * 128) + 1
    check(mf, ref.Case([70, 3], [200, 30], 8, 2, 128, page=64, base_page=base), 128)


@pytest.mark.parametrize("size", [0.0, 1e-30, 1e-6, 1e15, 1e20, 3e38])
def test_sizes_of_x(mf, size):
    """Rows of zeros, tiny rows, and rows whose squares' sum no float holds."""
    c = ref.Case([3, 20], [0, 7], 8, 2, 128)
    for x in (c.q, c.new_k):
        x.copy_((x / x.abs().amax(-1, keepdim=True).float() * size).to(x.dtype))
    if size == 3e38:
        c.q[0, 0] = 3e38  # every element as large as they come
    check(mf, c, 64)
    check(mf, c, 64, eps=2.0 ** -100)


def test_infinities_and_nan(mf):
    """An infinite element makes its head's others 0 and itself NaN, a NaN its head NaN; other heads are what they were."""
    c = ref.Case([2], [0], 4, 2, 64)
    qw, kw = weights(c)
    out = [torch.empty(2, 4, 64, dtype=c.q.dtype, device="cuda") for _ in range(2)]
    at, cache, norm = c.attn(mf), mf.kv_cache(c.k, c.v), mf.qk_norm(qw, kw, 1e-6)
    mf.mf_kv_append_norm(at, cache, c.step(mf), norm, c.new_k, c.new_v, c.q, out[0])
    c.q[0, 1, 5], c.q[1, 3, 0] = -math.inf, math.nan
    c.new_v[0, 0, 0] = math.nan  # a value is copied whatever it is
    mf.mf_kv_append_norm(at, cache, c.step(mf), norm, c.new_k, c.new_v, c.q, out[1])
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)
    a, b = out
    assert b[0, 1, 5].isnan() and (b[0, 1, :5] == 0).all() and (b[0, 1, 6:] == 0).all() and b[1, 3].isnan().all()
    b[0, 1], b[1, 3] = a[0, 1], a[1, 3]
    assert torch.equal(a, b)
    pg, ln = c.lines[0]
    assert torch.equal(c.v[pg, ln].view(torch.int16), c.new_v.contiguous().view(torch.int16))


def test_other_stream_and_graph(mf):
    """Captured behind other work on a stream of the caller's, replayed with other tokens and lengths."""
    c = ref.Case([2, 1], [300, 20], 8, 2, 128)
    at, cache, step = c.attn(mf), mf.kv_cache(c.k, c.v), c.step(mf)
    qw, kw = weights(c)
    norm, out, noise = mf.qk_norm(qw, kw, 1e-6), torch.empty(3, 8, 128, dtype=c.q.dtype, device="cuda"), torch.randn_like(c.q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def body():
        c.q.add_(noise)
        mf.mf_kv_append_norm(at, cache, step, norm, c.new_k, c.new_v, c.q, out)

    with torch.cuda.stream(s):
        body()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            body()
        for lens in ([302, 21], [5, 1], [77, 20]):
            c.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
            g.replay()
            s.synchronize()
            for got, x, w in ((out, c.q, qw), (torch.cat([c.k[a[n - m:n], b[n - m:n]] for (a, b), n, m in zip(c.lines, lens, c.new)]),
                                               c.new_k, kw)):
                want = norm64(x, w, 1e-6, 0.0)
                assert ((got.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -19) * want.abs()).all()
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)


def test_tokens_and_pages_that_are_not_there(mf):
    """Tokens of no sequence store nothing, a page outside the pool is never written; both are reported."""
    c = ref.Case([1, 3], [100, 7], 8, 2, 64)
    at = mf.mf_attn_create(mf.AttnShape(8, 2, 64, mf.MF_BF16), 2, c.tokens + 4, 0)
    norm = mf.qk_norm(*weights(c), 1e-6)
    q, k, v = (torch.cat((x[:2], x, x[:2])) for x in (c.q, c.new_k, c.new_v))
    kc, out = c.k.clone(), torch.empty(c.tokens + 4, 8, 64, dtype=c.q.dtype, device="cuda")
    mf.mf_kv_append_norm(at, mf.kv_cache(c.k, c.v), mf.step(c.q_start + 2, c.kv_len, c.pages, c.tokens + 4, 3), norm, k, v, q, out)
    assert mf.mf_attn_check(at) == mf.MF_E_INVAL and mf.mf_attn_check(at) == 0
    pg = torch.cat([a[n - m:n] for (a, b), n, m in zip(c.lines, c.len, c.new)])
    ln = torch.cat([b[n - m:n] for (a, b), n, m in zip(c.lines, c.len, c.new)])
    assert (c.k[pg, ln] != kc[pg, ln]).any()
    c.k[pg, ln] = kc[pg, ln]
    assert torch.equal(c.k.view(torch.int16), kc.view(torch.int16))
    for bad in (1 << 30, -3):
        c.pages[0, 100 // 16] = bad
        mf.mf_kv_append_norm(at, mf.kv_cache(c.k, c.v), c.step(mf), norm, c.new_k, c.new_v)
        assert mf.mf_attn_check(at) == mf.MF_E_INVAL
    mf.mf_attn_destroy(at)


def test_refusals(mf):
    c = ref.Case([3, 1], [10, 5], 8, 2, 64)
    at, cache, step, w = c.attn(mf), mf.kv_cache(c.k, c.v), c.step(mf), weights(c)
    good, out = mf.qk_norm(*w, 1e-6), torch.empty(4, 8, 64, dtype=c.q.dtype, device="cuda")
    for norm in (mf.qk_norm(*w, 0.0), mf.qk_norm(w[0].half(), None, 1e-6), mf.qk_norm(w[0][:32].contiguous(), None, 1e-6)):
        with pytest.raises(mf.MFError) as e:
            mf.mf_kv_append_norm(at, cache, step, norm, c.new_k, c.new_v, c.q, out)
        assert e.value.status == mf.MF_E_INVAL
    for kw in (dict(q=c.q[:3], q_out=out), dict(q=c.q, q_out=out.float()), dict(q=c.q), dict(q=c.q, q_out=out[:, :4])):
        with pytest.raises(mf.MFError) as e:
            mf.mf_kv_append_norm(at, cache, step, good, c.new_k, c.new_v, **kw)
        assert e.value.status == mf.MF_E_INVAL
    with pytest.raises(mf.MFError):
        mf.mf_kv_append_norm(at, cache, step, good, c.new_k[:, :1], c.new_v)
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)


# ---- prompts: from eight blocks an SM on (1216 tokens), four tokens a block

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, None), (128, 128), (128, 48), (256, 64), (256, 256)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_prompts(mf, dtype, d, rot, interleaved):
    """Sequences that begin and end inside a block's four tokens, a last block of three."""
    check(mf, ref.Case([700, 1, 0, 511, 2, 1, 408], [0, 200, 9, 100, 16, 3, 31], 6, 2, d, dtype, page=24), rot, interleaved, offset=1.0,
          w=[x - 1 for x in weights(ref.Case([1], [0], d=d, dtype=dtype))])


@pytest.mark.parametrize("tokens", [1215, 1216, 1217, 1218, 1219, 2432])
def test_prompts_of_any_length(mf, tokens):
    check(mf, ref.Case([tokens - 50, 50], [3, 70], 4, 2, 128, page=16), 128, in_place=True)
    check(mf, ref.Case([tokens], [0], 4, 2, 64, "f16", page=7), 64, with_q=False)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 5), (40, 8), (64, 4), (96, 32)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_heads_of_prompts(mf, hq, hkv, d):
    """Heads of several tokens in a warp, and in one round of a block's threads."""
    check(mf, ref.Case([1, 1218], [3, 0], hq, hkv, d), 64)


@pytest.mark.parametrize("sections", [(8, 12, 12), (0, 32), (11, 10, 6, 5)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_axes_of_prompts(mf, sections, interleaved):
    check(mf, ref.Case([7, 1300], [0, 5], 4, 4, 128, heads_first=True, row_pad=16), 64, interleaved, sections)


@pytest.mark.parametrize("page", [1, 64])
def test_single_tokens_of_many_sequences(mf, page):
    """Every token of a block has a sequence of its own."""
    check(mf, ref.Case([1] * 1301, [i % 50 for i in range(1301)], 4, 1, 128, page=page), 32)


@pytest.mark.parametrize("which", [(True, False), (False, True), (False, False)])
def test_prompts_with_one_norm_or_none(mf, which):
    for f32, rot in ((True, 128), (False, None)):
        c = ref.Case([1209, 9], [3, 64], 8, 2, 128)
        check(mf, c, rot, w=[x if yes else None for x, yes in zip(weights(c, f32), which)])


def test_sizes_of_x_in_prompts(mf):
    """Rows whose squares' sum no float holds beside ordinary ones and zeros, in one warp too."""
    c = ref.Case([1220], [0], 8, 2, 64)
    for x in (c.q, c.new_k):
        x[::3] = (x[::3] / x[::3].abs().amax(-1, keepdim=True).float() * 3e38).to(x.dtype)
        x[1::3, ::2] = 0
    check(mf, c, 64, eps=2.0 ** -100)


def test_offsets_of_prompts_beyond_32_bits(mf):
    base = 2 ** 31 // (64 * 2 * 128) + 1
    check(mf, ref.Case([1216, 3], [200, 30], 8, 2, 128, page=64, base_page=base), 128)


def test_prompt_tokens_and_pages_that_are_not_there(mf):
    """Tokens of no sequence, which share blocks with others, store no key and no value; nor does one whose page is outside the pool.  All
    others are right, and both are reported."""
    c = ref.Case([1, 1300], [100, 7], 8, 2, 64)
    norm, w = mf.qk_norm(*weights(c), 1e-6), weights(c)
    pg = torch.cat([a[n - m:n] for (a, b), n, m in zip(c.lines, c.len, c.new)])
    ln = torch.cat([b[n - m:n] for (a, b), n, m in zip(c.lines, c.len, c.new)])
    at = mf.mf_attn_create(mf.AttnShape(8, 2, 64, mf.MF_BF16), 2, c.tokens + 8, 0)

    def right(kc, vc, gone=None):
        keep = torch.ones(c.tokens, dtype=torch.bool, device="cuda")
        if gone is not None:
            keep[gone] = False
        want = norm64(c.new_k, w[1], 1e-6, 0.0)
        assert ((c.k[pg, ln].double() - want).abs() <= (2.0 ** -8 + 24 * 2.0 ** -24) * 1.01 * want.abs())[keep].all()
        assert torch.equal(c.v[pg, ln][keep], c.new_v[keep])
        for got, was in ((c.k, kc), (c.v, vc)):
            got[pg[keep], ln[keep]] = was[pg[keep], ln[keep]]
            assert torch.equal(got.view(torch.int16), was.view(torch.int16))

    kc, vc = c.k.clone(), c.v.clone()
    for before, after in ((2, 2), (5, 0), (0, 7)):
        q, k, v = (torch.cat((x[:before], x, x[:after])) for x in (c.q, c.new_k, c.new_v))
        out = torch.empty(before + c.tokens + after, 8, 64, dtype=c.q.dtype, device="cuda")
        step = mf.step(c.q_start + before, c.kv_len, c.pages, before + c.tokens + after, 1300)
        mf.mf_kv_append_norm(at, mf.kv_cache(c.k, c.v), step, norm, k, v, q, out)
        assert mf.mf_attn_check(at) == mf.MF_E_INVAL and mf.mf_attn_check(at) == 0
        right(kc, vc)
    page, bad = c.pages[1, 40].item(), (pg == c.pages[1, 40]).nonzero()[:, 0]
    for x in (1 << 30, -3):
        c.pages[1, 40] = x
        mf.mf_kv_append_norm(at, mf.kv_cache(c.k, c.v), c.step(mf), norm, c.new_k, c.new_v)
        assert mf.mf_attn_check(at) == mf.MF_E_INVAL
        right(kc, vc, bad)
    c.pages[1, 40] = page
    mf.mf_attn_destroy(at)


def test_prompts_on_another_stream_and_in_a_graph(mf):
    c = ref.Case([1250, 1], [300, 20], 8, 2, 128)
    at, cache, step = c.attn(mf), mf.kv_cache(c.k, c.v), c.step(mf)
    qw, kw = weights(c)
    norm, out, noise = mf.qk_norm(qw, kw, 1e-6), torch.empty_like(c.q.contiguous()), torch.randn_like(c.q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def body():
        c.q.add_(noise)
        mf.mf_kv_append_norm(at, cache, step, norm, c.new_k, c.new_v, c.q, out)

    with torch.cuda.stream(s):
        body()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            body()
        for lens in ([1550, 21], [1250, 1], [1401, 20]):
            c.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
            g.replay()
            s.synchronize()
            for got, x, w in ((out, c.q, qw), (torch.cat([c.k[a[n - m:n], b[n - m:n]] for (a, b), n, m in zip(c.lines, lens, c.new)]),
                                               c.new_k, kw)):
                want = norm64(x, w, 1e-6, 0.0)
                assert ((got.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -19) * want.abs()).all()
    assert mf.mf_attn_check(at) == 0
    mf.mf_attn_destroy(at)
