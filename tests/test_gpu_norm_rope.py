"""Norms of queries and keys with the rotation against the 64-bit form.

Tolerances. An output is one rounding to its type (half a step, HALF of the value) of an fp32 result. The fp32
result's relative error: a sum of squares walks at most 16 channels in each of 8 pieces and joins 6 times, each of
these operations off by 2^-24, so at most 134 2^-24, half of it in the root; rsq is off by 2^-23; then at most 4 products,
3 operations of the rotation and the tables' rounding: below 80 2^-24 < 2^-17, of |a| + |b| for a turned pair (a, b).
A gradient takes these errors on both of its terms, and the mean's own sum (again at most 134 2^-24): 2^-15 of the
sizes of its terms covers them. A weight's gradient adds at most 2^9 terms a lane here, and 1024 / 16 + 16 partial
sums: 2^-14 of the sum of the terms' sizes.
"""
import pytest

torch = pytest.importorskip("torch")
vc = pytest.importorskip("paper_2609_15810_amd")
import block_oracle as O  # noqa: E402

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16
EPS = 1e-5
NORMS = dict(none=vc.NORM_NONE, head=vc.NORM_HEAD, token=vc.NORM_TOKEN)
LAYOUTS = dict(none=vc.ROPE_NONE, interleaved=vc.ROPE_INTERLEAVED, half=vc.ROPE_HALF)


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    vc.lib()


class Problem:
    """Inputs on the CPU and the GPU: q and k from a packed projection [B, N, Hq + 2 Hk, d], outputs head-major"""

    def __init__(self, B, Hq, Hk, N, d, dtype, norm, layout, rot, grid=None, pos=False, weights=True, seed=0):
        g = torch.Generator().manual_seed(1000 * N + 10 * Hq + seed)
        self.__dict__.update(B=B, Hq=Hq, Hk=Hk, N=N, d=d, dtype=dtype, norm=norm, layout=layout, rot=rot, grid=grid)
        self.qkv = (torch.randn((B, N, Hq + 2 * Hk, d), generator=g) * 3 + 0.5).to(dtype)
        span = (lambda H: H * d) if norm == "token" else (lambda H: d)
        self.w = [(torch.randn(span(H), generator=g) if weights and norm != "none" else None) for H in (Hq, Hk)]
        self.dz = [torch.randn((B, H, N, d), generator=g).to(dtype) for H in (Hq, Hk)]
        self.pos = self.cos = self.sin = None
        c = s = torch.zeros((1, N, max(rot, 2) // 2), dtype=torch.float64)
        if layout != "none":
            if grid:
                ct, st = (torch.from_numpy(t) for t in vc.rope_tables_host(*grid))
                a = O.grid_angles(*grid)[None]
            else:
                rows = 40000 if pos else N + 3
                ct, st = (torch.from_numpy(t) for t in vc.rope_line_tables_host(rows, rot))
                at = torch.arange(N)[None]
                if pos:
                    at = torch.randint(0, rows, (B, N), generator=g)
                    at.view(-1)[0] = rows - 1
                    self.pos = at.to(torch.int32).cuda()
                a = O.angles(at, rot)
            self.cos, self.sin = ct.cuda(), st.cuda()
            c, s = a.cos(), a.sin()
        self.c, self.s = c, s
        self.op = vc.NormRope(B, Hq, Hk, N, d, norm=NORMS[norm], eps=EPS, layout=LAYOUTS[layout],
                              rot=rot if layout != "none" else None, grid=grid, dtype=dtype, training=True)
        dev = self.qkv.cuda()
        self.q, self.k = self.split(dev)
        if Hk == 0:
            self.k = None
        self.kw = dict(q_weight=None if self.w[0] is None else self.w[0].cuda(),
                       k_weight=None if self.w[1] is None or Hk == 0 else self.w[1].cuda(), cos=self.cos, sin=self.sin,
                       pos=self.pos)

    def split(self, packed):
        t = packed.transpose(1, 2)
        return t[:, :self.Hq], t[:, self.Hq:self.Hq + self.Hk]

    def new(self):
        return [torch.full((self.B, H, self.N, self.d), float("nan"), dtype=self.dtype, device="cuda") if H else None
                for H in (self.Hq, self.Hk)]

    def forward(self, out=None, **kw):
        out = out or self.new()
        self.op.forward(self.q, self.k, *out, **self.kw, **kw)
        return out

    def backward(self):
        """gradients into a packed buffer, its value part untouched"""
        dqkv = torch.full_like(self.qkv, 7.0).cuda()
        dq, dk = self.split(dqkv)
        dz = [t.cuda() for t in self.dz]
        dw = [None, None]
        if self.norm != "none":
            span = (lambda H: H * self.d) if self.norm == "token" else (lambda H: self.d)
            dw = [torch.full((span(H),), float("nan"), device="cuda") if H else None for H in (self.Hq, self.Hk)]
        self.op.backward(self.q, self.k, dz[0], dz[1] if self.Hk else None, dq, dk if self.Hk else None, dq_weight=dw[0],
                         dk_weight=dw[1], **self.kw)
        assert (dqkv[:, :, self.Hq + self.Hk:] == 7.0).all()
        return [dq, dk], dw

    def check(self, out, grads=None):
        half, tiny = O.HALF[self.dtype], O.TINY[self.dtype]
        for i, x in enumerate(self.split(self.qkv.double())):
            if x.shape[1] == 0:
                continue
            w = None if self.w[i] is None else self.w[i].double()
            ref = O.norm_rope(x, w, self.c, self.s, self.layout, self.rot, self.norm, EPS)
            size = O.pair_size(O.norm_rope(x, w, self.c, self.s, "none", 0, self.norm, EPS), self.layout, self.rot)
            err = (out[i].cpu().double() - ref).abs()
            assert (err <= half * (ref.abs() + 2.0 ** -17 * size) + 2.0 ** -17 * size + tiny).all(), float(err.max())
            if grads is None:
                continue
            dx, dw, dxs, dws = O.norm_rope_grad(x, w, self.c, self.s, self.layout, self.rot, self.norm, EPS,
                                                self.dz[i].double())
            err = (grads[0][i].cpu().double() - dx).abs()
            assert (err <= half * (dx.abs() + 2.0 ** -15 * dxs) + 2.0 ** -15 * dxs + tiny).all(), float(err.max())
            if dw is not None:
                err = (grads[1][i].cpu().double() - dw).abs()
                assert (err <= 2.0 ** -14 * dws).all(), float((err / dws).max())


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("norm,layout,rot", [("head", "interleaved", 128), ("head", "half", 128), ("token", "half", 64),
                                             ("token", "interleaved", 128), ("none", "half", 128), ("none", "half", 16),
                                             ("none", "interleaved", 112), ("head", "none", 0), ("token", "none", 0),
                                             ("head", "half", 112), ("head", "interleaved", 16)])
@pytest.mark.parametrize("B,Hq,Hk,N,pos", [(2, 12, 4, 37, True), (1, 3, 1, 130, False)])
def test_formats(dtype, norm, layout, rot, B, Hq, Hk, N, pos):
    p = Problem(B, Hq, Hk, N, 128, dtype, norm, layout, rot, pos=pos)
    p.check(p.forward(), p.backward())


@pytest.mark.parametrize("norm,layout,rot", [("head", "half", 64), ("token", "interleaved", 48), ("none", "half", 32),
                                             ("head", "none", 0)])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (5, 2), (16, 16), (40, 0)])
def test_heads_of_64(norm, layout, rot, Hq, Hk):
    p = Problem(2, Hq, Hk, 19, 64, BF, norm, layout, rot, pos=True)
    p.check(p.forward(), p.backward())


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("norm", ["head", "token", "none"])
def test_grid(norm, layout):
    p = Problem(2, 5, 3, 3 * 7 * 5, 128, BF, norm, layout, 128, grid=(3, 7, 5))
    p.check(p.forward(), p.backward())


@pytest.mark.parametrize("norm", ["head", "token"])
@pytest.mark.parametrize("B,Hq,Hk,N", [(1, 1, 1, 1), (1, 64, 64, 1), (1, 40, 8, 3), (3, 2, 2, 1), (1, 8, 8, 4097),
                                       (1, 1, 0, 6000), (1, 24, 1, 700)])
def test_sizes(norm, B, Hq, Hk, N):
    p = Problem(B, Hq, Hk, N, 128, BF, norm, "half", 128)
    p.check(p.forward(), p.backward())


def test_no_weights():
    p = Problem(1, 4, 2, 33, 128, BF, "head", "half", 128, weights=False)
    p.check(p.forward(), p.backward())


def test_zero_rows_and_infinities():
    p = Problem(1, 2, 2, 40, 128, BF, "head", "half", 128)
    p.qkv[0, 3] = 0.0
    p.q.copy_(p.split(p.qkv.cuda())[0])
    p.k.copy_(p.split(p.qkv.cuda())[1])
    p.check(p.forward(), p.backward())
    # an infinity or NaN spoils its own row only
    clean = [t.clone() for t in p.forward()]
    p.q[0, 1, 5, 17] = float("inf")
    p.k[0, 0, 6, 3] = float("nan")
    out = p.forward()
    for i, (h, n) in enumerate([(1, 5), (0, 6)]):
        assert not out[i][0, h, n].isfinite().all()
        keep = torch.ones_like(out[i], dtype=torch.bool)
        keep[0, h, n] = False
        assert torch.equal(out[i][keep], clean[i][keep])


@pytest.mark.parametrize("norm", ["head", "token", "none"])
def test_in_place(norm):
    p = Problem(2, 12, 4, 50, 128, BF, norm, "half", 64)
    ref = p.forward()
    grads, dw = p.backward()
    dz = [t.cuda() for t in p.dz]
    new = [None, None] if norm == "none" else [torch.empty_like(t) for t in dw]
    p.op.backward(p.q, p.k, *dz, *dz, dq_weight=new[0], dk_weight=new[1], **p.kw)
    p.op.forward(p.q, p.k, p.q, p.k, **p.kw)
    for a, b in zip([p.q, p.k] + dz, ref + grads):
        assert torch.equal(a, b)
    if norm != "none":
        assert torch.equal(new[0], dw[0]) and torch.equal(new[1], dw[1])


def test_shared_input_and_positions_out_of_range():
    # one row of queries for all tokens (stride 0), positions beyond the tables are clamped
    p = Problem(1, 4, 4, 60, 128, BF, "head", "half", 128, pos=True)
    one = p.q[:, :, :1].contiguous()
    p.qkv[:, :, :4] = one.cpu().transpose(1, 2)
    p.q = one.expand(1, 4, 60, 128)
    p.check(p.forward(), p.backward())
    p.pos[0, :2] = torch.tensor([-5, 1 << 30], dtype=torch.int32)
    out = p.forward()
    assert all(t.isfinite().all() for t in out)


def test_gradient_against_differences():
    """The loss sum(z dz) along a direction, by central differences of the forward kernel in fp16. A value of z is off
    by half a step, so the difference of two losses by at most 2 sum(|z| |dz|) 2^-11 / (2 h); h balances that against the
    third derivative."""
    p = Problem(1, 2, 1, 3, 64, FP, "token", "interleaved", 64)
    (dq, _), _ = p.backward()
    u = torch.randn(dq.shape, generator=torch.Generator().manual_seed(3)).cuda()
    q0, dz, h = p.q.clone(), p.dz[0].cuda().double(), 0.25
    loss, size, q = [], 0.0, []
    for s in (1.0, -1.0):
        p.q = (q0 + s * h * u).to(FP)
        q.append(p.q.double())
        z = p.forward()[0].double()
        loss.append((z * dz).sum())
        size = max(size, float((z * dz).abs().sum()))
    got, want = float((dq.double() * (q[0] - q[1])).sum()), float(loss[0] - loss[1])
    # the curvature's part: h^3 f''' of a function whose scale of change is |x| ~ 3: (0.25 / 3)^3 of its size
    assert abs(got - want) <= 2 * size * 2.0 ** -11 + (0.25 / 3.0) ** 3 * size


def test_wrong_tensors_refused():
    p = Problem(1, 4, 2, 33, 128, BF, "head", "half", 128)
    out = p.new()
    for q in (p.q.cpu(), p.q.half(), p.q[:, :3], p.q.transpose(2, 3).contiguous().transpose(2, 3)):
        with pytest.raises(vc.VcError):
            p.op.forward(q, p.k, *out, **p.kw)
    with pytest.raises(vc.VcError):
        p.op.forward(p.q, p.k, out[0], None, **p.kw)
    with pytest.raises(vc.VcError):
        p.op.forward(p.q, p.k, *out, **dict(p.kw, cos=p.cos[:, :32].contiguous()))
    with pytest.raises(vc.VcError):
        p.op.forward(p.q, p.k, *out, **dict(p.kw, q_weight=p.kw["q_weight"].half()))


def test_streams_and_graph():
    p = Problem(2, 12, 4, 210, 128, BF, "token", "half", 128)
    ref, (rg, rw) = p.forward(), p.backward()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = p.new()
    with torch.cuda.stream(s):
        p.forward(out)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, ref))
    out = p.forward(p.new(), stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, ref))
    dq, dk = (torch.empty_like(t) for t in rg)
    dw, dz = [torch.empty_like(t) for t in rw], [t.cuda() for t in p.dz]
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        p.op.forward(p.q, p.k, *out, **p.kw)
        p.op.backward(p.q, p.k, *dz, dq, dk, dq_weight=dw[0], dk_weight=dw[1], **p.kw)
    other = Problem(1, 3, 3, 500, 128, BF, "head", "half", 128)
    for _ in range(3):
        for t in out + [dq, dk] + dw:
            t.zero_()
        other.backward()
        torch.cuda.synchronize()
        g.replay()
        other.backward()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out + [dq, dk] + dw, ref + rg + rw))


@pytest.mark.parametrize("layout,rot", [("half", 32), ("half", 112), ("interleaved", 48)])
def test_channels_behind_the_turned_part_stay_as_they_are(layout, rot):
    p = Problem(1, 3, 2, 21, 128, FP, "none", layout, rot)
    p.q[0, 0, 4, rot + 1], p.q[0, 1, 5, 127], p.k[0, 0, 6, rot] = float("inf"), float("nan"), -0.0
    p.q[0, 2, 9, rot + 3] = -0.0
    bits = lambda t: t[..., rot:].contiguous().view(torch.int16)  # noqa: E731
    for x, z in zip((p.q, p.k), p.forward()):
        assert torch.equal(bits(x), bits(z))
        assert z[..., :rot].isfinite().all()


@pytest.mark.parametrize("norm", ["head", "token"])
@pytest.mark.parametrize("eps", [1e-30, 2.0 ** -126])
def test_small_eps(norm, eps):
    """1 / sqrt(eps) whose cube is beyond fp32: rows of zeros and ordinary ones (as check(), with this eps)"""
    p = Problem(1, 2, 1, 12, 128, BF, norm, "none", 0)
    p.q[:, :, 3] = 0.0
    p.op = vc.NormRope(1, 2, 1, 12, norm=NORMS[norm], eps=eps, layout=vc.ROPE_NONE, training=True)
    out, (grads, dw) = p.forward(), p.backward()
    eps = float(torch.tensor(eps))
    x, w, dz = p.q.cpu().double(), p.w[0].double(), p.dz[0].double()
    ref = O.norm_rope(x, w, p.c, p.s, "none", 0, norm, eps)
    assert ((out[0].cpu().double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -16) * ref.abs() + 2.0 ** -134).all()
    dx, dwr, dxs, dws = O.norm_rope_grad(x, w, p.c, p.s, "none", 0, norm, eps, dz)
    err = (grads[0].cpu().double() - dx).abs()
    assert (err <= 2.0 ** -8 * (dx.abs() + 2.0 ** -15 * dxs) + 2.0 ** -15 * dxs + 2.0 ** -134).all()
    assert ((dw[0].cpu().double() - dwr).abs() <= 2.0 ** -14 * dws).all()
