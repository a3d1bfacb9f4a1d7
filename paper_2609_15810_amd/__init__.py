"""Python binding of libvcattn.so, the MI355X (gfx950) 8-bit VC-Attention forward.

Argument marshalling only: every step of the attention path runs in the library's HIP kernels.
torch is used for device memory and the current stream. The names mirror the C ABI declared in
include/vc_attn.h (vc_attn_group, vc_attn_prep, vc_attn_forward, ...). There is no fallback: if
the shared library is missing, importing the entry points raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvcattn.so")
D = 128

VC_OK = 0
STATUS = {0: "VC_OK", 1: "VC_ERR_NULL", 2: "VC_ERR_SHAPE", 3: "VC_ERR_UNSUPPORTED", 4: "VC_ERR_WORKSPACE",
          5: "VC_ERR_ALIGN", 6: "VC_ERR_HIP", 7: "VC_ERR_INTERNAL"}
P_EXPCAST, P_EXP_THEN_CAST = 0, 1
QK_INT8, QK_FP8, QK_MXFP4 = 0, 1, 2
GROUP_IDENTITY, GROUP_CUBE, GROUP_KMEANS = 0, 1, 2
BF16, FP16 = 0, 1
NORM_NONE, NORM_HEAD, NORM_TOKEN = 0, 1, 2
ROPE_NONE, ROPE_INTERLEAVED, ROPE_HALF = 0, 1, 2
SCALE_NONE, SCALE_LINEAR, SCALE_BASE, SCALE_PARTS = 0, 1, 2, 3


class VcError(RuntimeError):
    def __init__(self, fn: str, status: int, lib=None):
        msg = f"{fn} returned {STATUS.get(status, status)}"
        if lib is not None:
            msg += f" ({lib.vc_status_str(status).decode()})"
            if status == 6:
                msg += f", hipError {lib.vc_last_hip_error()}"
        super().__init__(msg)
        self.status = status


class Shape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "H", "N", "d", "F", "Ht", "Wd")]


class Opts(C.Structure):
    _fields_ = [("qk_fmt", C.c_int32), ("p_mode", C.c_int32), ("rope", C.c_int32), ("hadamard", C.c_int32),
                ("smooth_k", C.c_int32), ("smooth_v", C.c_int32), ("sm_scale", C.c_float), ("beta", C.c_float)]


class GroupOpts(C.Structure):
    _fields_ = [("mode", C.c_int32), ("k", C.c_int32), ("iters", C.c_int32), ("warm_start", C.c_int32),
                ("cube", C.c_int32 * 3)]


class Prepped(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q", "q_scale", "k", "k_scale", "k_mean", "v", "v_scale", "v_mean",
                                          "q_mx_scale", "k_mx_scale")]


class View(C.Structure):
    _fields_ = [("data", C.c_void_p), ("sb", C.c_int64), ("sh", C.c_int64), ("sn", C.c_int64)]


_VIEW = C.c_char_p              # a view argument: the bytes of a View (made faster than the structure), or None
_pack_view = struct.Struct("4q").pack


class CrossShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "Hq", "Hk", "M", "N", "d")]


class CrossOpts(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("sm_scale", C.c_float), ("masked", C.c_int32)]


class NormRopeShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "Hq", "Hk", "N", "d")]


class NormRopeOpts(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("norm", C.c_int32), ("layout", C.c_int32), ("rot", C.c_int32),
                ("eps", C.c_float), ("rows", C.c_int32), ("F", C.c_int32), ("Ht", C.c_int32), ("Wd", C.c_int32)]


class RopeScaling(C.Structure):
    _fields_ = [("kind", C.c_int32)] + [(n, C.c_double) for n in ("factor", "trained", "fast", "slow", "magnitude")]


_lib = None


def lib():
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2609_15810_amd/build.py "
                               "(the HIP library is required; there is no fallback)")
        L = C.CDLL(LIB_PATH)
        L.vc_attn_workspace_size.restype = C.c_size_t
        L.vc_attn_workspace_size.argtypes = [C.POINTER(Shape), C.POINTER(Opts), C.POINTER(GroupOpts)]
        L.vc_status_str.restype = C.c_char_p
        L.vc_status_str.argtypes = [C.c_int]
        L.vc_last_hip_error.restype = C.c_int
        L.vc_rope_tables.restype = C.c_int
        L.vc_rope_tables.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_double, C.c_void_p, C.c_void_p]
        L.vc_attn_group.restype = C.c_int
        L.vc_attn_group.argtypes = [C.POINTER(Shape), C.POINTER(GroupOpts), C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.vc_attn_prep.restype = C.c_int
        L.vc_attn_prep.argtypes = [C.POINTER(Shape), C.POINTER(Opts), C.c_void_p, C.c_void_p, C.c_void_p,
                                   C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(Prepped),
                                   C.c_void_p, C.c_size_t, C.c_void_p]
        L.vc_attn_prep_noalloc.restype = C.c_int
        L.vc_attn_prep_noalloc.argtypes = [C.POINTER(Shape), C.POINTER(Opts), C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(Prepped),
                                           C.c_void_p]
        L.vc_attn_forward.restype = C.c_int
        L.vc_attn_forward.argtypes = [C.POINTER(Shape), C.POINTER(Opts), C.POINTER(Prepped), C.c_void_p,
                                      C.c_void_p, C.c_void_p]
        L.vc_attn_forward_codes.restype = C.c_int
        L.vc_attn_forward_codes.argtypes = [C.POINTER(Shape), C.POINTER(Opts), C.POINTER(Prepped), C.c_void_p,
                                            C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.vc_fp8_score_product.restype = C.c_int
        L.vc_fp8_score_product.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.vc_cross_attn_workspace_size.restype = C.c_size_t
        L.vc_cross_attn_workspace_size.argtypes = [C.POINTER(CrossShape), C.POINTER(CrossOpts), C.c_int32]
        p = C.c_void_p
        L.vc_cross_attn_forward.restype = C.c_int
        L.vc_cross_attn_forward.argtypes = [p, p] + [_VIEW] * 3 + [p, p, C.c_int64, _VIEW, p] + [p, C.c_size_t, p]
        L.vc_cross_attn_backward.restype = C.c_int
        L.vc_cross_attn_backward.argtypes = [p, p] + [_VIEW] * 3 + [p, p, C.c_int64, _VIEW, p] + [_VIEW] * 4 + \
            [p, C.c_size_t, p]
        L.vc_norm_rope_workspace_size.restype = C.c_size_t
        L.vc_norm_rope_workspace_size.argtypes = [C.POINTER(NormRopeShape), C.POINTER(NormRopeOpts)]
        L.vc_norm_rope.restype = C.c_int
        L.vc_norm_rope.argtypes = [p, p] + [_VIEW] * 2 + [p] * 5 + [_VIEW] * 2 + [p]
        L.vc_norm_rope_backward.restype = C.c_int
        L.vc_norm_rope_backward.argtypes = [p, p] + [_VIEW] * 2 + [p] * 5 + [_VIEW] * 4 + [p, p, p, C.c_size_t, p]
        L.vc_rope_line_tables.restype = C.c_int
        L.vc_rope_line_tables.argtypes = [C.c_int32, C.c_int32, C.c_double, C.POINTER(RopeScaling), C.c_void_p,
                                          C.c_void_p]
        L.vc_opts_default.argtypes = [C.POINTER(Opts)]
        L.vc_group_opts_default.argtypes = [C.POINTER(GroupOpts)]
        _lib = L
    return _lib


def _check(fn: str, st: int):
    if st != VC_OK:
        raise VcError(fn, st, lib())


def make_shape(B: int, H: int, grid) -> Shape:
    F, Ht, Wd = grid
    return Shape(B, H, F * Ht * Wd, D, F, Ht, Wd)


def make_opts(p_mode=P_EXPCAST, rope=True, hadamard=True, smooth_k=True, smooth_v=True, sm_scale=0.0,
              beta=-0.35, qk_fmt=QK_INT8) -> Opts:
    o = Opts()
    lib().vc_opts_default(C.byref(o))
    o.qk_fmt = int(qk_fmt)
    o.p_mode, o.rope, o.hadamard = int(p_mode), int(rope), int(hadamard)
    o.smooth_k, o.smooth_v, o.sm_scale, o.beta = int(smooth_k), int(smooth_v), float(sm_scale), float(beta)
    return o


def make_group_opts(mode=GROUP_KMEANS, k=32, iters=8, warm_start=False, cube=(4, 2, 16)) -> GroupOpts:
    g = GroupOpts()
    lib().vc_group_opts_default(C.byref(g))
    g.mode, g.k, g.iters, g.warm_start = int(mode), int(k), int(iters), int(bool(warm_start))
    g.cube[0], g.cube[1], g.cube[2] = (int(c) for c in cube)
    return g


def workspace_size(shape: Shape, opts: Opts | None = None, gopts: GroupOpts | None = None) -> int:
    return int(lib().vc_attn_workspace_size(C.byref(shape), C.byref(opts) if opts is not None else None,
                                            C.byref(gopts) if gopts is not None else None))


def rope_tables_host(F: int, Ht: int, Wd: int, theta: float = 10000.0):
    """vc_rope_tables into host numpy arrays [(F+Ht+Wd), 64] fp32."""
    cos_t = np.empty((F + Ht + Wd, 64), np.float32)
    sin_t = np.empty_like(cos_t)
    _check("vc_rope_tables", lib().vc_rope_tables(F, Ht, Wd, float(theta), cos_t.ctypes.data, sin_t.ctypes.data))
    return cos_t, sin_t


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


@dataclass
class PreppedBuffers:
    """Device buffers of the low-bit operands (layouts documented in include/vc_attn.h)."""
    q: object
    q_scale: object
    k: object
    k_scale: object
    k_mean: object
    v: object
    v_scale: object
    v_mean: object
    q_mx_scale: object = None
    k_mx_scale: object = None

    def as_struct(self) -> Prepped:
        return Prepped(*(None if t is None else t.data_ptr()
                         for t in (self.q, self.q_scale, self.k, self.k_scale, self.k_mean, self.v, self.v_scale,
                                   self.v_mean, self.q_mx_scale, self.k_mx_scale)))


def alloc_prepped(shape: Shape, device="cuda", qk_fmt: int = None) -> PreppedBuffers:
    """Buffers for vc_attn_prep / vc_attn_forward. INT8 and FP8: q, k [B, H, Np, 128] bytes and fp32
    block scales; MXFP4: q, k packed codes [B, H, Np, 64] bytes and E8M0 scale bytes [B, H, Np, 4]."""
    import torch
    B, H, N = shape.B, shape.H, shape.N
    T = (N + 127) // 128
    Np = 128 * T
    e = dict(device=device)
    mx = qk_fmt == QK_MXFP4
    cw = D // 2 if mx else D
    return PreppedBuffers(
        q=torch.empty((B, H, Np, cw), dtype=torch.int8, **e), q_scale=torch.empty((B, H, T), dtype=torch.float32, **e),
        k=torch.empty((B, H, Np, cw), dtype=torch.int8, **e), k_scale=torch.empty((B, H, T), dtype=torch.float32, **e),
        k_mean=torch.empty((B, H, D), dtype=torch.float32, **e),
        v=torch.empty((B, H, Np, D), dtype=torch.uint8, **e), v_scale=torch.empty((B, H, D), dtype=torch.float32, **e),
        v_mean=torch.empty((B, H, T, D), dtype=torch.int16, **e),
        q_mx_scale=torch.empty((B, H, Np, 4), dtype=torch.uint8, **e) if mx else None,
        k_mx_scale=torch.empty((B, H, Np, 4), dtype=torch.uint8, **e) if mx else None)


def vc_attn_group(shape, gopts, V, centroids, labels, perm, inv_perm, ws, stream=None):
    _check("vc_attn_group", lib().vc_attn_group(C.byref(shape), C.byref(gopts), _ptr(V), _ptr(centroids),
                                                _ptr(labels), _ptr(perm), _ptr(inv_perm), _ptr(ws),
                                                ws.numel() * ws.element_size() if ws is not None else 0,
                                                _stream(stream)))


def vc_attn_prep(shape, opts, Q, K, V, perm, q_perm, rope_cos, rope_sin, out: PreppedBuffers, ws, stream=None):
    st = out.as_struct()
    _check("vc_attn_prep", lib().vc_attn_prep(C.byref(shape), C.byref(opts), _ptr(Q), _ptr(K), _ptr(V), _ptr(perm),
                                              _ptr(q_perm), _ptr(rope_cos), _ptr(rope_sin), C.byref(st), _ptr(ws),
                                              ws.numel() * ws.element_size(), _stream(stream)))


def vc_attn_prep_noalloc(shape, opts, Q, K, V, perm, q_perm, rope_cos, rope_sin, out: PreppedBuffers, stream=None):
    st = out.as_struct()
    _check("vc_attn_prep_noalloc", lib().vc_attn_prep_noalloc(C.byref(shape), C.byref(opts), _ptr(Q), _ptr(K), _ptr(V),
                                                              _ptr(perm), _ptr(q_perm), _ptr(rope_cos), _ptr(rope_sin),
                                                              C.byref(st), _stream(stream)))


def vc_attn_forward(shape, opts, inp: PreppedBuffers, q_perm, O, stream=None):
    st = inp.as_struct()
    _check("vc_attn_forward", lib().vc_attn_forward(C.byref(shape), C.byref(opts), C.byref(st), _ptr(q_perm),
                                                    _ptr(O), _stream(stream)))


def vc_attn_forward_codes(shape, opts, inp: PreppedBuffers, q_perm, O, p_codes, stream=None):
    st = inp.as_struct()
    nbytes = p_codes.numel() * p_codes.element_size() if p_codes is not None else 0
    _check("vc_attn_forward_codes", lib().vc_attn_forward_codes(C.byref(shape), C.byref(opts), C.byref(st),
                                                                _ptr(q_perm), _ptr(O), _ptr(p_codes), nbytes,
                                                                _stream(stream)))


def vc_fp8_score_product(a, b, c_in, out, stream=None):
    """a, b: uint8 E4M3 bytes [n, 32, 128]; c_in, out: fp32 [n, 32, 32] (device tensors)."""
    n = a.shape[0]
    _check("vc_fp8_score_product", lib().vc_fp8_score_product(_ptr(a), _ptr(b), _ptr(c_in), _ptr(out), n,
                                                              _stream(stream)))


class Attention:
    """Buffers for one attention shape and the three calls of the path.

    group() computes the permutation (and centroids) from V; prep() produces the low-bit
    operands; forward() writes O. Inputs are bf16 tensors [B, H, N, 128] on the device
    (torch.bfloat16 or int16 bit patterns).
    """

    def __init__(self, B, H, grid, opts: Opts | None = None, gopts: GroupOpts | None = None, device="cuda"):
        import torch
        self.shape = make_shape(B, H, grid)
        self.opts = opts if opts is not None else make_opts()
        self.gopts = gopts if gopts is not None else make_group_opts()
        self.device = device
        ws = workspace_size(self.shape, self.opts, self.gopts)
        if ws == 0:
            raise VcError("vc_attn_workspace_size", 2)
        self.ws = torch.empty(ws, dtype=torch.uint8, device=device)
        N = self.shape.N
        e = dict(device=device, dtype=torch.int32)
        self.perm = torch.empty((B, H, N), **e)
        self.inv_perm = torch.empty((B, H, N), **e)
        self.labels = torch.empty((B, H, N), **e)
        self.centroids = torch.zeros((B, H, max(self.gopts.k, 1), D), dtype=torch.float32, device=device)
        self.prepped = alloc_prepped(self.shape, device, self.opts.qk_fmt)
        cos_t, sin_t = rope_tables_host(*grid)
        self.rope_cos = torch.from_numpy(cos_t).to(device)
        self.rope_sin = torch.from_numpy(sin_t).to(device)

    def group(self, V, warm_start=None, stream=None):
        g = self.gopts
        if warm_start is not None:
            g = make_group_opts(g.mode, g.k, g.iters, warm_start, tuple(g.cube))
        vc_attn_group(self.shape, g, V, self.centroids, self.labels, self.perm, self.inv_perm, self.ws, stream)

    def prep(self, Q, K, V, perm="own", q_perm=None, stream=None):
        p = self.perm if isinstance(perm, str) else perm
        vc_attn_prep(self.shape, self.opts, Q, K, V, p, q_perm, self.rope_cos, self.rope_sin, self.prepped, self.ws,
                     stream)

    def forward(self, O, q_perm=None, stream=None):
        vc_attn_forward(self.shape, self.opts, self.prepped, q_perm, O, stream)

    def forward_codes(self, O, p_codes, q_perm=None, stream=None):
        """forward() that also writes the probability codes, uint8 [B, H, N, 128 T] (debugging)."""
        vc_attn_forward_codes(self.shape, self.opts, self.prepped, q_perm, O, p_codes, stream)


# ---- operators around the attention --------------------------------------------------------------

def make_rope_scaling(kind=SCALE_NONE, factor=1.0, trained=4096, fast=32.0, slow=1.0, magnitude=0.0) -> RopeScaling:
    return RopeScaling(int(kind), float(factor), float(trained), float(fast), float(slow), float(magnitude))


def rope_line_tables_host(rows: int, rot: int = D, theta: float = 10000.0, scaling: RopeScaling | None = None):
    """vc_rope_line_tables into host numpy arrays [rows, rot/2] fp32."""
    cos_t = np.empty((max(rows, 0), max(rot, 0) // 2), np.float32)
    sin_t = np.empty_like(cos_t)
    _check("vc_rope_line_tables", lib().vc_rope_line_tables(
        rows, rot, float(theta), C.byref(scaling) if scaling is not None else None, cos_t.ctypes.data,
        sin_t.ctypes.data))
    return cos_t, sin_t


def _device(device):
    import torch
    d = torch.device(device)
    return torch.device(d.type, torch.cuda.current_device()) if d.type == "cuda" and d.index is None else d


class _Operator:
    """What the operators around the attention have in common. Each tensor is checked against its shape, type and
    device (the library sees addresses only); VcError is raised as for a refusal of the library. A call runs on the
    device of its tensors, on the given stream or that device's current one."""

    def __init__(self, dtype, device):
        import torch
        types = {torch.bfloat16: BF16, torch.float16: FP16}
        if dtype not in types:
            raise VcError(type(self).__name__, 3, lib())
        self.dtype, self.device = dtype, _device(device)
        self.c_dtype = types[dtype]
        self.ws = None
        self._f32, self._i32 = torch.float32, torch.int32
        self._current_device, self._current_stream = torch.cuda.current_device, torch._C._cuda_getCurrentRawStream

    def _refuse(self, status):
        raise VcError(type(self).__name__, status, lib())

    def _view(self, t, shape):
        """a tensor in any strides whose channels are contiguous"""
        if t is None:
            return None
        if t.shape != shape or t.dtype != self.dtype or t.device != self.device:
            self._refuse(2)
        sb, sh, sn, sc = t.stride()
        if sc != 1:
            self._refuse(5)
        return _pack_view(t.data_ptr(), sb, sh, sn)

    def _flat(self, t, shape, dtype):
        """a contiguous tensor"""
        if t is None:
            return None
        if t.shape != shape or t.dtype != dtype or t.device != self.device:
            self._refuse(2)
        if not t.is_contiguous():
            self._refuse(5)
        return t.data_ptr()

    def _call(self, fn, stream, *args):
        index = self.device.index
        s = self._current_stream(index) if stream is None else stream.cuda_stream
        if self._current_device() == index:
            st = getattr(lib(), fn)(*args, s)
        else:
            import torch
            with torch.cuda.device(self.device):
                st = getattr(lib(), fn)(*args, s)
        if st != VC_OK:
            raise VcError(fn, st, lib())


class NormRope(_Operator):
    """Norms of queries and keys with the rotation by position, for one shape: vc_norm_rope and its gradients.

    Tensors are [B, heads, N, d] of `dtype` in any strides whose channels are contiguous (a transposed view of
    a packed projection). grid: (frames, rows, columns) with the tables of vc_rope_tables; None: positions on a line
    with [rows, rot/2] tables. training: hold the workspace of the weights' gradients. Two calls that overlap in
    time (on two streams, or two captured graphs) need an object each: backward() uses the object's workspace.
    """

    def __init__(self, B, Hq, Hk, N, d=D, norm=NORM_HEAD, eps=1e-6, layout=ROPE_INTERLEAVED, rot=None, grid=None,
                 dtype=None, training=False, device="cuda"):
        import torch
        super().__init__(torch.bfloat16 if dtype is None else dtype, device)
        self.shape = NormRopeShape(B, Hq, Hk, N, d)
        self.rot = 0 if layout == ROPE_NONE else (d if rot is None else rot)
        # the tables' rows are known with the tables; 1 stands for them in the checks here
        self.opts = self._opts(norm, layout, eps, 1, grid)
        size = lib().vc_norm_rope_workspace_size(C.byref(self.shape), C.byref(self.opts))
        if size == C.c_size_t(-1).value:
            raise VcError("vc_norm_rope_workspace_size", 2, lib())
        if training:
            self.ws = torch.empty(max(size, 16), dtype=torch.uint8, device=self.device)
        self._q, self._k = (B, Hq, N, d), (B, Hk, N, d)
        span = (lambda H: (H * d,)) if norm == NORM_TOKEN else (lambda H: (d,))
        self._qw, self._kw, self._pos = span(Hq), span(Hk), (B, N)
        self._norm, self._layout, self._eps, self._grid = norm, layout, eps, grid
        self._c_shape = C.byref(self.shape)

    def _opts(self, norm, layout, eps, rows, grid):
        return NormRopeOpts(self.c_dtype, norm, layout, self.rot, eps, rows, *(grid or (0, 0, 0)))

    def _inputs(self, q, k, q_weight, k_weight, cos, sin, pos):
        if self.shape.Hk == 0 and (k is not None or k_weight is not None):
            self._refuse(2)
        opts = self.opts
        if self._layout != ROPE_NONE:
            if cos is None or sin is None:
                self._refuse(1)
            rows = sum(self._grid) if self._grid else len(cos)
            table = (rows, self.rot // 2)
            cos, sin = self._flat(cos, table, self._f32), self._flat(sin, table, self._f32)
            if not self._grid:
                opts = self._opts(self._norm, self._layout, self._eps, rows, None)
        else:
            cos = sin = None
        return (self._c_shape, C.byref(opts), self._view(q, self._q), self._view(k, self._k),
                self._flat(q_weight, self._qw, self._f32), self._flat(k_weight, self._kw, self._f32), cos, sin,
                self._flat(pos, self._pos, self._i32))

    def forward(self, q, k, q_out, k_out, q_weight=None, k_weight=None, cos=None, sin=None, pos=None, stream=None):
        """q_out, k_out = the normed and turned q, k (k and k_out None with Hk = 0)."""
        self._call("vc_norm_rope", stream, *self._inputs(q, k, q_weight, k_weight, cos, sin, pos),
                   self._view(q_out, self._q), self._view(k_out, self._k))

    def backward(self, q, k, dq_out, dk_out, dq, dk, q_weight=None, k_weight=None, dq_weight=None, dk_weight=None,
                 cos=None, sin=None, pos=None, stream=None):
        """dq, dk (and dq_weight, dk_weight where given) = the gradients of q, k and of the weights."""
        self._call("vc_norm_rope_backward", stream, *self._inputs(q, k, q_weight, k_weight, cos, sin, pos),
                   self._view(dq_out, self._q), self._view(dk_out, self._k), self._view(dq, self._q),
                   self._view(dk, self._k), self._flat(dq_weight, self._qw, self._f32),
                   self._flat(dk_weight, self._kw, self._f32), None if self.ws is None else self.ws.data_ptr(),
                   0 if self.ws is None else self.ws.numel())


class CrossAttention(_Operator):
    """Attention to the states of another sequence for one shape: vc_cross_attn_forward and its gradients.

    Q, O (and dO, dQ) are [B, Hq, M, d], K, V (dK, dV) [B, Hk, N, d] of `dtype` in any strides whose channels
    are contiguous. k_len: int32 [B]; k_mask (with masked=True): uint8 or bool [B, N], nonzero where a key counts.
    training: also hold the workspace of backward(). Two calls that overlap in time (on two streams, or two captured
    graphs) need an object each: both calls use the object's workspace.
    """

    def __init__(self, B, Hq, Hk, M, N, d=D, dtype=None, sm_scale=0.0, masked=False, training=False, device="cuda"):
        import torch
        super().__init__(torch.bfloat16 if dtype is None else dtype, device)
        self.shape = CrossShape(B, Hq, Hk, M, N, d)
        self.opts = CrossOpts(self.c_dtype, sm_scale, int(bool(masked)))
        self._c = C.byref(self.shape), C.byref(self.opts)
        size = 0
        for backward in range(2 if training else 1):
            need = lib().vc_cross_attn_workspace_size(*self._c, backward)
            if need == C.c_size_t(-1).value:
                raise VcError("vc_cross_attn_workspace_size", 2, lib())
            size = max(size, need)
        self.ws = torch.empty(max(size, 16), dtype=torch.uint8, device=self.device)
        self._ws = self.ws.data_ptr(), self.ws.numel()
        self._q, self._k, self._b, self._mask, self._lse = (B, Hq, M, d), (B, Hk, N, d), (B,), (B, N), (B, Hq, M)
        self._mask_types = (torch.uint8, torch.bool)

    def _inputs(self, Q, K, V, k_len, k_mask, O, lse):
        mask, stride = None, 0
        if k_mask is not None:
            if k_mask.shape != self._mask or k_mask.dtype not in self._mask_types or k_mask.device != self.device:
                self._refuse(2)
            stride, s = k_mask.stride()
            if s != 1 and self.shape.N > 1:
                self._refuse(5)
            mask = k_mask.data_ptr()
        return (*self._c, self._view(Q, self._q), self._view(K, self._k), self._view(V, self._k),
                self._flat(k_len, self._b, self._i32), mask, stride, self._view(O, self._q),
                self._flat(lse, self._lse, self._f32))

    def forward(self, Q, K, V, O, lse=None, k_len=None, k_mask=None, stream=None):
        """O = softmax(sm_scale Q K^T) V; lse [B, Hq, M] fp32 is written where given (for backward)."""
        self._call("vc_cross_attn_forward", stream, *self._inputs(Q, K, V, k_len, k_mask, O, lse), *self._ws)

    def backward(self, Q, K, V, O, lse, dO, dQ, dK, dV, k_len=None, k_mask=None, stream=None):
        """dQ, dK, dV from dO, with O (or None: it is not read) and lse as forward() wrote them (training=True)."""
        self._call("vc_cross_attn_backward", stream, *self._inputs(Q, K, V, k_len, k_mask, O, lse),
                   self._view(dO, self._q), self._view(dQ, self._q), self._view(dK, self._k), self._view(dV, self._k),
                   *self._ws)
