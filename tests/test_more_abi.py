"""What of the append with norms, attention over shared lines and verification is decided on the host: struct layouts and refusals.
Addresses are made up: a call that is refused touches nothing."""
import ctypes
import math

import pytest

AT = 1 << 20  # an aligned address


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_09686_gb300 as pkg
    return pkg


def changed(s, **kw):
    t = type(s).from_buffer_copy(s)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


@pytest.fixture(scope="module")
def handle(mf):
    """The beginning of an attention handle: shape, the most sequences and tokens."""
    class Handle(ctypes.Structure):
        _fields_ = [("shape", mf.AttnShape), ("max_seqs", ctypes.c_int32), ("max_tokens", ctypes.c_int32), ("rest", ctypes.c_uint8 * 488)]
    return ctypes.pointer(Handle(mf.AttnShape(8, 2, 64, mf.MF_BF16), 4, 64))


def test_struct_layouts(mf):
    assert [ctypes.sizeof(t) for t in (mf.QkNorm, mf.Shared, mf.Cuts, mf._VerifyArgs)] == [32, 24, 32, 184]


def parts(mf):
    return (mf.KvCache(AT, AT, 8192, 512, 64, 10, 16), mf.Step(None, AT, AT, 2, 2, 1, 5), mf.QkNorm(AT, AT, 1e-6, 0.0, mf.MF_BF16, 0),
            mf.Rope(AT, AT, None, 100, 64, 0, 1), mf._AppendArgs(AT, AT, AT, AT, 512, 128, 128, 512))


def test_append_norm_refusals(mf, handle):
    cache, step, norm, rope, args = parts(mf)

    def refused(handle=handle, cache=cache, step=step, norm=norm, rope=rope, args=args):
        assert mf._lib.mf_kv_append_norm(ctypes.cast(handle, ctypes.c_void_p), cache, step, norm, rope, args, None) == mf.MF_E_INVAL

    refused(handle=None)
    refused(norm=None)
    refused(args=None)
    for kw in (dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(eps=2.0 ** -101), dict(offset=math.nan),
               dict(offset=math.inf), dict(dtype=mf.MF_F16), dict(dtype=7), dict(q_weight=AT + 2), dict(k_weight=AT + 8)):
        refused(norm=changed(norm, **kw))
    for kw in (dict(k=None), dict(v=AT + 2), dict(q_out=None), dict(q_stride=7), dict(k_stride=-8)):
        refused(args=changed(args, **kw))
    for kw in (dict(rot_dim=24), dict(rot_dim=128), dict(n_pos=0), dict(n_axes=5), dict(cos=None)):
        refused(rope=changed(rope, **kw))
    for kw in (dict(n_seqs=5), dict(n_tokens=65), dict(kv_len=None), dict(max_q=0)):
        refused(step=changed(step, **kw))
    refused(cache=changed(cache, page_size=0))
    assert mf._lib.mf_kv_append_norm(ctypes.cast(handle, ctypes.c_void_p), cache, changed(step, n_tokens=0, n_seqs=0), norm, rope, args,
                                     None) == mf.MF_OK


def test_shared_refusals(mf, handle):
    cache, step, *_ = parts(mf)
    args = mf._AttnArgs(AT, AT, AT, 512, 512, 0.1, 0, 1, 0)
    group = mf.Shared(AT, AT, 1, 0)

    def status(handle=handle, step=step, group=group, args=args):
        return mf._lib.mf_attn_forward_shared(ctypes.cast(handle, ctypes.c_void_p), cache, step, group, args, None)

    assert status() == mf.MF_E_STATE  # mf_attn_share was not called
    for kw in (dict(handle=None), dict(group=None), dict(args=None)):
        assert status(**kw) == mf.MF_E_INVAL
    for kw in (dict(first=None), dict(len=None), dict(first=AT + 2), dict(n_groups=-1)):
        assert status(group=changed(group, **kw)) == mf.MF_E_INVAL
    for kw in (dict(window=1), dict(window=-1), dict(scale=0.0), dict(q=None), dict(out=AT + 4), dict(lse=AT + 1)):
        assert status(args=changed(args, **kw)) == mf.MF_E_INVAL
    assert status(step=changed(step, n_seqs=5)) == mf.MF_E_INVAL
    for n in (0, -1, (1 << 20) + 1):
        assert mf._lib.mf_attn_share(ctypes.cast(handle, ctypes.c_void_p), n) == mf.MF_E_INVAL
    assert mf._lib.mf_attn_share(None, 1) == mf.MF_E_INVAL


def test_verify_refusals(mf):
    none = mf.Cuts()
    good = mf._VerifyArgs(AT, AT, AT, AT, AT, AT, none, none, AT, AT, AT, AT, 1000, 1000, 1000, 2, 6, 1000, mf.MF_F32)
    for kw in (dict(logits=None), dict(row_start=None), dict(tokens=None), dict(u=None), dict(noise=None), dict(token=None),
               dict(accepted=None), dict(work=None), dict(work=AT + 8), dict(logits=AT + 2), dict(draft_logits=AT + 1), dict(noise=AT + 2),
               dict(u=AT + 1), dict(tokens=AT + 2), dict(token=AT + 2), dict(accepted=AT + 2), dict(logprob=AT + 2), dict(row_start=AT + 2),
               dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(dtype=8), dict(n_seqs=-1), dict(n_rows=-1), dict(n_seqs=0),
               dict(logits_stride=999), dict(draft_stride=999), dict(noise_stride=999), dict(n_rows=(1 << 26) + 1),
               dict(cuts=mf.Cuts(AT + 2)), dict(draft_cuts=mf.Cuts(None, None, None, AT + 1))):
        assert mf._lib.mf_verify(changed(good, **kw), None) == mf.MF_E_INVAL, kw
    assert mf._lib.mf_verify(None, None) == mf.MF_E_INVAL
    assert mf._lib.mf_verify(changed(good, n_seqs=0, n_rows=0), None) == mf.MF_OK


def test_verify_bytes(mf):
    sizes = [mf.mf_verify_bytes(2, n, 1000) for n in (0, 1, 7, 1000)]
    assert 0 < sizes[0] <= sizes[1] < sizes[2] < sizes[3]
    for a in ((-1, 1, 10), (1, -1, 10), (1, 1, 0), (1, 1, (1 << 20) + 1), (1, (1 << 26) + 1, 10)):
        with pytest.raises(mf.MFError) as e:
            mf.mf_verify_bytes(*a)
        assert e.value.status == mf.MF_E_INVAL


def test_descriptions_refuse_what_is_not_on_the_gpu(mf):
    torch = pytest.importorskip("torch")
    w, i = torch.ones(64), torch.zeros(2, dtype=torch.int32)
    for make in (lambda: mf.qk_norm(w, w, 1e-6), lambda: mf.shared(i, i[:1]), lambda: mf.cuts(temperature=w)):
        with pytest.raises(ValueError):
            make()
    for bad in ((w, w[:32]), (w, w.half()), (w[::2], w[::2]), (w.view(8, 8), None), (w.double(), None)):
        with pytest.raises(ValueError):
            mf.qk_norm(*bad, 1e-6)
    for bad in ((i, i), (i.long(), i[:1].long()), (i.view(1, 2), i[:1])):
        with pytest.raises(ValueError):
            mf.shared(*bad)
    for bad in (dict(temperature=w.double()), dict(top_k=w), dict(top_p=w[::2]), dict(min_p=w.view(8, 8))):
        with pytest.raises(ValueError):
            mf.cuts(**bad)
    x = torch.zeros(2, 10)
    with pytest.raises(mf.MFError) as e:
        mf.mf_verify(x, i, i, w[:2], x[:1], i, i, torch.zeros(4096, dtype=torch.uint8))
    assert e.value.status == mf.MF_E_INVAL


class OnGpu:
    """What the binding asks of a tensor, on a GPU that this machine need not have."""
    is_cuda = True

    def __init__(self, dtype, *shape, device=0):
        self.dtype, self.shape, self.at = dtype, shape, device

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        s = tuple(math.prod(self.shape[k + 1:]) for k in range(len(self.shape)))
        return s if i is None else s[i]

    def numel(self):
        return math.prod(self.shape)

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def is_pinned(self):
        return False

    def get_device(self):
        return self.at

    def data_ptr(self):
        return AT


def test_verify_refuses_tensors_of_another_gpu(mf, monkeypatch):
    """Every tensor of a call, settings too, has to be on the current device: the kernels would read another's addresses as their own."""
    torch = pytest.importorskip("torch")
    if not mf._Types.codes:
        mf._Types.load()
    calls = []
    monkeypatch.setattr(mf._Types, "device", lambda: 0)
    monkeypatch.setattr(mf, "_stream", lambda s: None)
    monkeypatch.setattr(mf._lib, "mf_verify", lambda a, s: calls.append(a) or mf.MF_OK)
    f32, i32, n, seqs, v = torch.float32, torch.int32, 5, 2, 300
    good = dict(logits=(f32, n, v), draft_logits=(f32, n, v), noise=(f32, seqs, v), row_start=(i32, seqs + 1), tokens=(i32, n), u=(f32, n),
                token=(i32, n), accepted=(i32, seqs), logprob=(f32, n), work=(torch.uint8, mf.mf_verify_bytes(seqs, n, v)))
    sets = dict(temperature=(f32, seqs), top_k=(i32, seqs), top_p=(f32, seqs), min_p=(f32, seqs))

    def call(other=None):
        args = {k: OnGpu(*a, device=int(k == other)) for k, a in good.items()}
        for which in ("cuts", "draft_cuts"):
            args[which] = mf.cuts(**{k: OnGpu(*a, device=int((which, k) == other)) for k, a in sets.items()})
        mf.mf_verify(**args)

    call()
    assert len(calls) == 1
    for other in list(good) + [(w, k) for w in ("cuts", "draft_cuts") for k in sets]:
        with pytest.raises(mf.MFError) as e:
            call(other)
        assert e.value.status == mf.MF_E_INVAL
    assert len(calls) == 1
