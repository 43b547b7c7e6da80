"""What of the attention and sampling entry points is decided on the host: struct layouts, K(n), refusals."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def mf():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_09686_gb300 as pkg
    return pkg


def test_struct_layouts(mf):
    assert [ctypes.sizeof(t) for t in (mf.AttnShape, mf.KvCache, mf.Step, mf.Rope)] == [16, 48, 40, 56]


@pytest.mark.parametrize("n,page", [(0, 16), (1, 16), (16, 16), (17, 16), (4096, 64), (1000, 7)])
def test_kv_bytes(mf, n, page):
    lines = (n + page - 1) // page * page
    for hq, hkv, d, dt in ((32, 8, 128, mf.MF_BF16), (16, 1, 256, mf.MF_F16)):
        assert mf.mf_kv_bytes(mf.AttnShape(hq, hkv, d, dt), 48, n, page) == 48 * lines * hkv * d * 2 * 2


def test_kv_bytes_enter_the_plan(mf):
    kv = mf.mf_kv_bytes(mf.AttnShape(16, 2, 256, mf.MF_BF16), 48, 32768, 64)
    m = mf.Model(48, 2048, 128, 8, 768, mf.Q8_0)
    free, full = (mf.mf_plan(m, mf.PlanReq(35.0, 1 << 40, 0, b, 64, 0)) for b in (0, kv))
    assert full.lower_bound_bytes - free.lower_bound_bytes == kv


@pytest.mark.parametrize("shape", [(8, 3, 64, 1), (8, 0, 64, 1), (0, 1, 64, 1), (8, 2, 96, 1), (8, 2, 64, 0), (8, 2, 64, 8),
                                   (129, 1, 64, 1)])
def test_bad_shapes(mf, shape):
    for call in (lambda: mf.mf_kv_bytes(mf.AttnShape(*shape), 1, 1, 1), lambda: mf.mf_attn_create(mf.AttnShape(*shape), 1, 1, 0)):
        with pytest.raises(mf.MFError) as e:
            call()
        assert e.value.status == mf.MF_E_INVAL


def test_bad_sizes(mf):
    s = mf.AttnShape(8, 2, 64, mf.MF_F16)
    for a in ((0, 1, 16), (1, -1, 16), (1, 1, 0), (2 ** 31 - 1, 2 ** 62, 2 ** 31 - 1)):
        with pytest.raises(mf.MFError) as e:
            mf.mf_kv_bytes(s, *a)
        assert e.value.status == mf.MF_E_INVAL
    for a in ((0, 1, 0), (1, 0, 0), (1, 1, -1)):
        with pytest.raises(mf.MFError) as e:
            mf.mf_attn_create(s, *a)
        assert e.value.status == mf.MF_E_INVAL
    mf.mf_attn_destroy(None)
