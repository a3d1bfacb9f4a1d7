"""Norms with the rotation, without a GPU: refusals of the C ABI, and the host tables."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2609_15810_amd as vc

FAKE = 0x10000  # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def L():
    return vc.lib()


def shape(B=2, Hq=4, Hk=2, N=60, d=128):
    return vc.NormRopeShape(B, Hq, Hk, N, d)


def opts(dtype=vc.BF16, norm=vc.NORM_HEAD, layout=vc.ROPE_INTERLEAVED, rot=128, eps=1e-6, rows=60, grid=(0, 0, 0)):
    return vc.NormRopeOpts(dtype, norm, layout, rot, eps, rows, *grid)


def view(s, H, data=FAKE, **kw):
    st = dict(sb=s.N * H * s.d, sh=s.d, sn=H * s.d)
    st.update(kw)
    return vc.View(data, st["sb"], st["sh"], st["sn"])


def forward(L, s, o, q=None, out=None, pos=None, cos=FAKE, k="own", weight=None):
    q = q or view(s, s.Hq)
    kv = view(s, max(s.Hk, 1)) if k == "own" else k
    ref = lambda v: None if v is None else bytes(v)  # noqa: E731
    return L.vc_norm_rope(C.byref(s), C.byref(o), ref(q), ref(kv), weight, None, cos, FAKE, pos,
                          ref(out or view(s, s.Hq)), ref(kv), None)


def backward(L, s, o, ws=FAKE, ws_bytes=1 << 40, dw=FAKE, q="own"):
    q = view(s, s.Hq) if q == "own" else q
    v, k = view(s, s.Hq), view(s, max(s.Hk, 1))
    r = lambda t: None if t is None else bytes(t)  # noqa: E731
    return L.vc_norm_rope_backward(C.byref(s), C.byref(o), r(q), r(k), None, None, FAKE, FAKE, None, r(v), r(k), r(v),
                                   r(k), dw, None, ws, ws_bytes, None)


@pytest.mark.parametrize("kw", [dict(B=0), dict(N=0), dict(Hq=0), dict(Hk=-1), dict(d=96), dict(d=256),
                                dict(B=1 << 16, N=1 << 16), dict(Hq=16384)])
def test_shapes_refused(L, kw):
    s = shape(**kw)
    assert forward(L, s, opts(norm=vc.NORM_HEAD)) == 2
    assert L.vc_norm_rope_workspace_size(C.byref(s), C.byref(opts())) == C.c_size_t(-1).value


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(norm=3), dict(norm=-1), dict(layout=3), dict(rot=0), dict(rot=24),
                                dict(rot=144), dict(eps=0.0), dict(eps=1e-39), dict(eps=math.nan), dict(eps=math.inf), dict(rows=0),
                                dict(grid=(4, 0, 0)), dict(norm=vc.NORM_NONE, layout=vc.ROPE_NONE, rot=0),
                                dict(layout=vc.ROPE_NONE)])
def test_options_refused(L, kw):
    assert forward(L, shape(), opts(**kw)) == 3


def test_other_refusals(L):
    s, o = shape(), opts()
    assert forward(L, shape(Hq=65), opts(norm=vc.NORM_TOKEN)) == 2            # more than 8192 channels under one norm
    assert forward(L, s, opts(grid=(3, 4, 6))) == 2                           # 72 tokens, not 60
    far = shape(B=1, N=1 << 25)                                               # rows of the tables beyond 32-bit indexes
    assert forward(L, far, opts(grid=(1 << 25, 1, 1))) == 2
    assert forward(L, shape(d=64), opts(rot=64, grid=(3, 4, 5))) == 3         # the grid's tables are for 128 channels
    assert forward(L, s, opts(grid=(3, 4, 5)), pos=FAKE) == 3
    assert forward(L, s, opts(rows=59)) == 2                                  # fewer rows than tokens
    assert forward(L, s, o, cos=None) == 1
    assert forward(L, s, o, cos=FAKE + 4) == 5
    assert forward(L, s, o, pos=FAKE + 2) == 5
    assert forward(L, s, o, k=None) == 1
    assert forward(L, s, o, weight=FAKE + 4) == 5
    assert forward(L, s, o, q=view(s, 4, data=None)) == 1
    assert forward(L, s, o, q=view(s, 4, data=FAKE + 8)) == 5
    assert forward(L, s, o, q=view(s, 4, sn=516)) == 5
    assert forward(L, s, o, q=view(s, 4, sn=-512)) == 2
    assert forward(L, s, o, q=view(s, 4, sb=1 << 41)) == 2
    # outputs whose rows overlap: shared along an axis, or closer than a row is long
    assert forward(L, s, o, out=view(s, 4, sb=0)) == 2
    assert forward(L, s, o, out=view(s, 4, sn=0)) == 2
    assert forward(L, s, o, out=view(s, 4, sh=120)) == 2
    assert forward(L, s, o, out=view(s, 4, sn=504)) == 2
    # the stride of an axis of extent 1 is not looked at
    assert forward(L, shape(B=1), o, out=view(shape(B=1), 4, sb=-3), cos=None) == 1


def test_backward_refusals(L):
    s, o = shape(), opts()
    size = L.vc_norm_rope_workspace_size(C.byref(s), C.byref(o))
    assert 0 < size <= 2 * 128 * 4 * 120 and size % (2 * 128 * 4) == 0   # rows of two weights of 128, for 120 tokens
    assert backward(L, s, o, ws=None) == 4
    assert backward(L, s, o, ws_bytes=size - 1) == 4
    assert backward(L, s, o, ws=FAKE + 8) == 5
    assert backward(L, s, o, dw=FAKE + 4) == 5
    assert backward(L, s, o, q=None) == 1
    assert backward(L, s, opts(norm=vc.NORM_NONE)) == 3   # no weights, so no gradient of them


def test_line_tables_plain():
    c, s = vc.rope_line_tables_host(70000, 64)
    for p in (0, 1, 777, 69999):
        ang = p * 10000.0 ** (-2.0 * np.arange(32) / 64)
        # one rounding to fp32 of a value at most 1
        assert np.abs(c[p] - np.cos(ang)).max() <= 2.0 ** -25 + 1e-15
        assert np.abs(s[p] - np.sin(ang)).max() <= 2.0 ** -25 + 1e-15


def frequencies(scaling, rot=128):
    """read back from row 1 (angles below pi for all pairs)"""
    c, s = vc.rope_line_tables_host(2, rot, 10000.0, scaling)
    return np.arctan2(s[1].astype(np.float64), c[1].astype(np.float64))


def test_line_tables_scaled():
    base = 10000.0 ** (-2.0 * np.arange(64) / 128)
    close = lambda a, b: np.abs(a / b - 1.0).max() < 1e-6  # noqa: E731  (two fp32 roundings)
    assert close(frequencies(None), base)
    assert close(frequencies(vc.make_rope_scaling()), base)
    assert close(frequencies(vc.make_rope_scaling(vc.SCALE_LINEAR, 8.0)), base / 8.0)
    f = frequencies(vc.make_rope_scaling(vc.SCALE_BASE, 8.0))
    assert close(f[:1], base[:1]) and close(f[-1:], base[-1:] / 8.0) and close(f[1:] / f[:-1], np.full(63, f[1] / f[0]))
    f = frequencies(vc.make_rope_scaling(vc.SCALE_PARTS, 8.0, trained=4096, fast=32.0, slow=1.0))
    turns = 4096 * base / (2 * np.pi)
    keep = np.clip((turns - 1.0) / 31.0, 0.0, 1.0)
    assert 0 < (keep == 1).sum() < 64 and (keep == 0).sum() > 0
    assert close(f, base * keep + base / 8.0 * (1.0 - keep))
    c, s = vc.rope_line_tables_host(5, 64, 10000.0, vc.make_rope_scaling(vc.SCALE_LINEAR, 2.0, magnitude=1.25))
    assert np.abs(np.hypot(c, s) - 1.25).max() < 2e-7


@pytest.mark.parametrize("kw", [dict(kind=4), dict(kind=1, factor=0.5), dict(kind=1, factor=math.inf),
                                dict(kind=0, magnitude=-1.0), dict(kind=3, factor=2.0, trained=0.0),
                                dict(kind=3, factor=2.0, fast=1.0, slow=1.0), dict(kind=2, factor=math.nan)])
def test_scaling_refused(kw):
    with pytest.raises(vc.VcError) as e:
        vc.rope_line_tables_host(4, 64, 10000.0, vc.make_rope_scaling(**kw))
    assert e.value.status == 3


@pytest.mark.parametrize("rows,rot,theta", [(0, 64, 1e4), (4, 24, 1e4), (4, 0, 1e4), (4, 144, 1e4), (4, 64, 0.0),
                                            (4, 64, math.nan)])
def test_tables_refused(rows, rot, theta):
    with pytest.raises(vc.VcError) as e:
        vc.rope_line_tables_host(rows, rot, theta)
    assert e.value.status == 2
