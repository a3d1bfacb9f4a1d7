"""Attention to another sequence, without a GPU: refusals of the C ABI and workspace sizes."""
import ctypes as C
import math

import pytest

import paper_2609_15810_amd as vc

FAKE = 0x10000  # never dereferenced: every call below fails validation first
INVALID = C.c_size_t(-1).value


@pytest.fixture(scope="module")
def L():
    return vc.lib()


def shape(B=2, Hq=4, Hk=2, M=50, N=30, d=128):
    return vc.CrossShape(B, Hq, Hk, M, N, d)


def opts(dtype=vc.BF16, sm_scale=0.0, masked=0):
    return vc.CrossOpts(dtype, sm_scale, masked)


def view(H, n, d=128, data=FAKE, **kw):
    st = dict(sb=n * H * d, sh=d, sn=H * d)
    st.update(kw)
    return vc.View(data, st["sb"], st["sh"], st["sn"])


def views(s, **kw):
    q, k = view(s.Hq, s.M, s.d), view(s.Hk, s.N, s.d)
    return dict(dict(Q=q, K=k, V=k, O=q, dO=q, dQ=q, dK=k, dV=k), **kw)


def forward(L, s, o, k_len=None, k_mask=None, stride=None, lse=FAKE, ws=FAKE, ws_bytes=1 << 40, **kw):
    v = {n: (None if t is None else bytes(t)) for n, t in views(s, **kw).items()}
    return L.vc_cross_attn_forward(C.byref(s), C.byref(o), v["Q"], v["K"], v["V"], k_len, k_mask,
                                   s.N if stride is None else stride, v["O"], lse, ws, ws_bytes, None)


def backward(L, s, o, k_mask=None, lse=FAKE, ws=FAKE, ws_bytes=1 << 40, **kw):
    v = {n: (None if t is None else bytes(t)) for n, t in views(s, **kw).items()}
    return L.vc_cross_attn_backward(C.byref(s), C.byref(o), v["Q"], v["K"], v["V"], None, k_mask, s.N, v["O"], lse,
                                    v["dO"], v["dQ"], v["dK"], v["dV"], ws, ws_bytes, None)


BAD = vc.View(None, 0, 0, 0)


@pytest.mark.parametrize("kw", [dict(B=0), dict(Hq=0), dict(Hk=0), dict(M=0), dict(N=0), dict(d=96), dict(d=32),
                                dict(Hq=3), dict(B=1 << 20, M=1 << 10), dict(B=1 << 20, N=1 << 10),
                                dict(Hk=1, B=1, M=(1 << 28) + 1), dict(Hq=1, Hk=1, B=1, N=(1 << 30) + 1),
                                dict(B=1 << 23, M=1, N=1), dict(B=1 << 22, Hq=1, Hk=1, M=1, N=1)])
def test_shapes_refused(L, kw):
    s = shape(**kw)
    assert forward(L, s, opts()) == 2 and backward(L, s, opts()) == 2
    for b in (0, 1):
        assert L.vc_cross_attn_workspace_size(C.byref(s), C.byref(opts()), b) == INVALID


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(dtype=-1), dict(sm_scale=-1.0), dict(sm_scale=math.nan),
                                dict(sm_scale=math.inf), dict(sm_scale=3e38), dict(masked=2)])
def test_options_refused(L, kw):
    assert forward(L, shape(), opts(**kw)) == 3 and backward(L, shape(), opts(**kw)) == 3


@pytest.mark.parametrize("name", ["Q", "K", "V", "O"])
def test_views_refused(L, name):
    s, o = shape(), opts()
    H, n = (4, 50) if name in "QO" else (2, 30)
    assert forward(L, s, o, **{name: None}) == 1
    assert forward(L, s, o, **{name: BAD}) == 1
    assert forward(L, s, o, **{name: view(H, n, data=FAKE + 8)}) == 5
    assert forward(L, s, o, **{name: view(H, n, sn=H * 128 + 4)}) == 5
    assert forward(L, s, o, **{name: view(H, n, sh=-128)}) == 2
    assert forward(L, s, o, **{name: view(H, n, sb=1 << 41)}) == 2


@pytest.mark.parametrize("name", ["O", "dO", "dQ", "dK", "dV"])
def test_backward_views_refused(L, name):
    s, o = shape(), opts()
    H, n = (2, 30) if name in ("dK", "dV") else (4, 50)
    if name != "O":
        assert backward(L, s, o, **{name: None}) == 1
    assert backward(L, s, o, **{name: BAD}) == 1
    assert backward(L, s, o, **{name: view(H, n, data=FAKE + 8)}) == 5
    if name[0] == "d" and name != "dO":   # outputs whose rows overlap
        assert backward(L, s, o, **{name: view(H, n, sh=0)}) == 2
        assert backward(L, s, o, **{name: view(H, n, sb=0)}) == 2


def test_other_refusals(L):
    s, o, m = shape(), opts(), opts(masked=1)
    assert forward(L, s, o, O=view(4, 50, sn=0)) == 2
    assert forward(L, s, o, O=view(4, 50, sn=504)) == 2
    assert forward(L, s, o, k_len=FAKE + 2) == 5
    assert forward(L, s, o, lse=FAKE + 2) == 5
    assert forward(L, s, o, k_mask=FAKE) == 3
    assert forward(L, s, m) == 1
    assert forward(L, s, m, k_mask=FAKE, stride=29) == 2
    assert forward(L, s, m, k_mask=FAKE, ws=None) == 4
    assert backward(L, s, o, lse=None) == 1
    assert backward(L, s, o, lse=FAKE + 1) == 5
    for b, call in ((0, lambda w: forward(L, s, m, k_mask=FAKE, ws_bytes=w)),
                    (1, lambda w: backward(L, s, m, k_mask=FAKE, ws_bytes=w))):
        size = L.vc_cross_attn_workspace_size(C.byref(s), C.byref(m), b)
        assert 0 < size < 1 << 30
        assert call(size - 1) == 4
    assert forward(L, s, m, k_mask=FAKE, ws=FAKE + 8) == 5


def test_workspace_sizes(L):
    # a full grid of rows with no mask needs none; the backward pass always keeps its rows' statistics
    s = shape(B=1, Hq=12, Hk=12, M=32760, N=512)
    assert L.vc_cross_attn_workspace_size(C.byref(s), C.byref(opts()), 0) == 0
    assert L.vc_cross_attn_workspace_size(C.byref(s), C.byref(opts()), 1) >= 12 * 32760 * 8
    # split keys leave a part each: rows of d fp32 and two statistics
    s = shape(B=1, Hq=2, Hk=2, M=10, N=10000)
    assert L.vc_cross_attn_workspace_size(C.byref(s), C.byref(opts()), 0) >= 2 * 2 * 10 * (128 + 2) * 4
