"""Attention to another sequence and its gradients against the 64-bit form, within the bounds that block_oracle.Cross
derives from the roundings that the kernels make."""
import pytest

torch = pytest.importorskip("torch")
vc = pytest.importorskip("paper_2609_15810_amd")
import block_oracle as O  # noqa: E402

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    vc.lib()


class Problem:
    """Q, O, dO, dQ as views of token-major tensors, K, V and their gradients of packed ones; guards around outputs"""

    def __init__(self, B, Hq, Hk, M, N, d=128, dtype=BF, mask="none", scale=0.0, packed=True, gain=1.5, seed=0):
        g = torch.Generator().manual_seed(100 * M + N + seed)
        self.B, self.Hq, self.Hk, self.M, self.N, self.d, self.dtype = B, Hq, Hk, M, N, d, dtype
        rand = lambda *s, f=1.0: (torch.randn(s, generator=g) * f).to(dtype)  # noqa: E731
        q, kv, do = rand(B, M, Hq, d, f=gain), rand(B, N, 2, Hk, d, f=1.2), rand(B, M, Hq, d)
        self.valid = torch.ones((B, N), dtype=torch.bool)
        self.kw = {}
        if mask in ("len", "both"):
            # from all keys to none; one length beyond the keys
            k_len = torch.tensor([N + 5 if b == 0 else N * (B - 1 - b) // max(B - 1, 1) for b in range(B)])
            self.valid &= torch.arange(N)[None] < k_len[:, None]
            self.kw["k_len"] = k_len.to(torch.int32).cuda()
        if mask in ("mask", "both"):
            on = torch.rand((B, N), generator=g) < torch.linspace(0.8, 0.1, B)[:, None]
            if B > 1:
                on[-1] = False
            self.valid &= on
            self.kw["k_mask"] = on.to(torch.uint8).mul(3).cuda()
        # what does not count may hold anything
        kv[~self.valid] = float("nan")
        self.cpu = [t.transpose(1, 2) for t in (q, kv[:, :, 0], kv[:, :, 1], do)]
        dev = [t.cuda() for t in (q, kv, do)]
        self.Q, self.K, self.V = dev[0].transpose(1, 2), dev[1][:, :, 0].transpose(1, 2), dev[1][:, :, 1].transpose(1, 2)
        self.dO = dev[2].transpose(1, 2)
        if not packed:
            self.Q, self.K, self.V, self.dO = (t.contiguous() for t in (self.Q, self.K, self.V, self.dO))
        self.scale = scale
        self.op = vc.CrossAttention(B, Hq, Hk, M, N, d, dtype=dtype, sm_scale=scale, masked="k_mask" in self.kw,
                                    training=True)

    def guarded(self, B, H, n):
        """[B, H, n, d] inside a wider token-major buffer of sevens, and a check that the rest stayed"""
        buf = torch.full((B, n + 3, H + 1, self.d), 7.0, dtype=self.dtype, device="cuda")
        view = buf[:, 1:n + 1, :H].transpose(1, 2)

        def intact():
            keep = torch.ones_like(buf, dtype=torch.bool)
            keep[:, 1:n + 1, :H] = False
            return bool((buf[keep] == 7.0).all())
        return view, intact

    def forward(self, **kw):
        out, intact = self.guarded(self.B, self.Hq, self.M)
        lse = torch.full((self.B, self.Hq, self.M), float("nan"), device="cuda")
        self.op.forward(self.Q, self.K, self.V, out, lse, **self.kw, **kw)
        torch.cuda.synchronize()
        assert intact()
        return out, lse

    def backward(self, out, lse, **kw):
        made = [self.guarded(self.B, H, n) for H, n in ((self.Hq, self.M), (self.Hk, self.N), (self.Hk, self.N))]
        grads = [m[0] for m in made]
        self.op.backward(self.Q, self.K, self.V, out, lse, self.dO, *grads, **self.kw, **kw)
        torch.cuda.synchronize()
        assert all(m[1]() for m in made)
        return grads

    def check(self, backward=True):
        out, lse = self.forward()
        q, k, v, do = self.cpu
        ref = O.Cross(q, k, v, self.valid, self.dtype, self.scale, do if backward else None)
        near(out, ref.O, ref.O_err, "O")
        lse = lse.cpu().double()
        empty = ref.lse == -float("inf")
        assert torch.equal(lse == -float("inf"), empty)
        assert ((lse - ref.lse)[~empty].abs() <= ref.lse_err.expand_as(lse)[~empty]).all()
        if backward:
            for name, got in zip(("dQ", "dK", "dV"), self.backward(out, lse.float().cuda())):
                near(got, getattr(ref, name), getattr(ref, name + "_err"), name)


def near(got, ref, err, name):
    got = got.cpu().double()
    assert got.isfinite().all(), name
    bad = (got - ref).abs() > err
    assert not bad.any(), (name, int(bad.sum()), float(((got - ref).abs() / err.clamp(min=1e-300)).max()))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("mask", ["none", "len", "mask", "both"])
@pytest.mark.parametrize("B,Hq,Hk,M,N", [(3, 4, 2, 130, 100), (2, 3, 3, 33, 257)])
def test_formats(dtype, d, mask, B, Hq, Hk, M, N):
    Problem(B, Hq, Hk, M, N, d, dtype, mask).check()


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("B,Hq,Hk,M,N", [
    (1, 1, 1, 1, 1), (2, 2, 1, 1, 2), (1, 1, 1, 700, 1), (1, 2, 2, 1, 700),          # one query, one key
    (1, 2, 2, 31, 63), (1, 2, 2, 32, 64), (1, 2, 2, 33, 65), (1, 2, 2, 128, 128), (1, 1, 1, 129, 129),   # tile edges
    (1, 8, 1, 5, 40), (2, 7, 1, 37, 300), (1, 40, 40, 3, 20),                        # groups of heads
    (1, 1, 1, 3001, 77), (16, 2, 2, 200, 64)])
def test_sizes(packed, B, Hq, Hk, M, N):
    Problem(B, Hq, Hk, M, N, packed=packed).check()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,Hq,Hk,M,N,mask", [(1, 8, 2, 1, 3000, "none"), (2, 4, 4, 40, 4100, "mask"),
                                              (3, 2, 1, 16, 2500, "len"), (1, 32, 8, 1, 1500, "both")])
def test_split_keys(dtype, B, Hq, Hk, M, N, mask):
    Problem(B, Hq, Hk, M, N, 128, dtype, mask).check()


@pytest.mark.parametrize("d", [128, 64])
def test_split_rows(d):
    Problem(1, 2, 1, 4001, 130, d).check()
    Problem(2, 2, 2, 2100, 40, d, mask="mask").check()


def test_many_rows_at_once():
    """the whole grid of a call of several thousand workgroups, on sampled rows"""
    p = Problem(1, 12, 12, 32760, 512)
    out, lse = p.forward()
    at = torch.cat([torch.arange(200), torch.arange(16300, 16500), torch.arange(32560, 32760)])
    q, k, v, _ = p.cpu
    ref = O.Cross(q[:, :, at], k, v, p.valid, BF)
    near(out[:, :, at.cuda()], ref.O, ref.O_err, "O")


@pytest.mark.parametrize("B,Hq,Hk,M,N,d,dtype,mask", [
    (2, 12, 4, 2900, 130, 128, BF, "both"),     # grouped heads, ragged lists, an item without a key
    (1, 24, 24, 2817, 64, 128, FP, "none"),     # one tile a block
    (3, 8, 8, 2570, 201, 64, BF, "len"), (2, 16, 2, 2305, 1, 64, FP, "none"), (4, 40, 40, 300, 70, 128, BF, "mask"),
    (1, 300, 300, 257, 65, 64, BF, "none")])
def test_blocks_of_many_rows(B, Hq, Hk, M, N, d, dtype, mask):
    """enough blocks of 256 rows for the kernel that walks over them: ends of heads, of blocks and of the work of a CU"""
    Problem(B, Hq, Hk, M, N, d, dtype, mask).check(backward=False)


@pytest.mark.parametrize("scale", [0.02, 0.5])
def test_scale(scale):
    Problem(1, 2, 2, 50, 90, scale=scale).check()


def test_peaked_rows():
    # scores of several hundred: the softmax takes one key, the running maximum moves over the tiles
    Problem(1, 2, 2, 70, 400, gain=60.0).check(backward=False)


def test_shared_operands():
    # one set of encoder states for all items, one row of queries for all places
    p = Problem(3, 2, 2, 40, 70)
    p.K, p.V = p.K[:1].expand(3, 2, 70, 128), p.V[:1].expand(3, 2, 70, 128)
    p.Q = p.Q[:, :, :1].expand(3, 2, 40, 128)
    q, k, v, do = p.cpu
    p.cpu = [q[:, :, :1].expand(3, 2, 40, 128), k[:1].expand(3, 2, 70, 128), v[:1].expand(3, 2, 70, 128), do]
    p.check()


def test_offsets_beyond_32_bits():
    p = Problem(1, 1, 1, 40, 5)
    far = torch.empty(4 * (1 << 30) + 128, dtype=BF, device="cuda")   # rows 2 GiB apart
    k = far.as_strided((1, 1, 5, 128), (8, 8, 1 << 30, 1))
    k.copy_(p.K)
    p.K = k
    p.check()
    out = far.as_strided((1, 1, 5, 128), (8, 8, 1 << 30, 1))
    q5 = p.Q[:, :, :5]
    op = vc.CrossAttention(1, 1, 1, 5, 5)
    near_o = torch.empty((1, 1, 5, 128), dtype=BF, device="cuda")
    kk = p.K.contiguous()
    op.forward(q5, kk, p.V, near_o)
    op.forward(q5, kk, p.V, out)
    assert torch.equal(out, near_o)


def test_rows_far_apart():
    # strides of queries and of their gradients that one buffer does not reach over a tile
    p = Problem(1, 2, 1, 70, 40)
    ref, lse = p.forward()
    grads = p.backward(ref, lse)
    wide = torch.empty((3, 70, 1 << 22), dtype=BF, device="cuda")
    far = [wide[i].as_strided((1, 2, 70, 128), (256, 128, 1 << 22, 1), wide[i].storage_offset()) for i in range(3)]
    far[0].copy_(p.Q)
    far[1].copy_(p.dO)
    p.Q, p.dO = far[0], far[1]
    out, lse2 = p.forward()
    assert torch.equal(out, ref) and torch.equal(lse2, lse)
    far[2].copy_(out)
    assert all(torch.equal(a, b) for a, b in zip(p.backward(far[2], lse), grads))


def test_reproducible():
    p = Problem(2, 4, 2, 1000, 300, mask="mask")
    out, lse = p.forward()
    grads = p.backward(out, lse)
    for _ in range(3):
        again, lse2 = p.forward()
        assert torch.equal(again, out) and torch.equal(lse2, lse)
        assert all(torch.equal(a, b) for a, b in zip(p.backward(out, lse), grads))


def test_values_that_are_not_finite():
    # an infinite value of a key that counts reaches the rows of its head, and nothing else
    p = Problem(1, 2, 2, 40, 100)
    clean, _ = p.forward()
    clean = clean.clone()
    p.V[0, 1, 99, 5] = float("inf")
    out, _ = p.forward()
    assert torch.equal(out[0, 0], clean[0, 0])
    assert (out[0, 1, :, 5] == float("inf")).all()
    keep = torch.arange(128, device="cuda") != 5
    assert torch.equal(out[0, 1][:, keep], clean[0, 1][:, keep])
    # a NaN in a query spoils its own row
    p.V[0, 1, 99, 5] = 0.0
    clean, _ = p.forward()
    clean = clean.clone()
    p.Q[0, 0, 7, 3] = float("nan")
    out, _ = p.forward()
    assert out[0, 0, 7].isnan().all()
    rows = torch.arange(40, device="cuda") != 7
    assert torch.equal(out[:, :, rows], clean[:, :, rows])


@pytest.mark.parametrize("B,H,M,N", [(1, 2, 40, 200), (4, 40, 300, 200), (1, 2, 3, 4000)])
def test_scores_of_minus_infinity(B, H, M, N):
    # keys whose scores are -inf take no part; a row all of whose scores are -inf has no softmax (NaN), and the rows
    # that the same waves work on next are not touched by it
    p = Problem(B, H, H, M, N)
    p.Q.abs_()
    p.cpu[0] = p.cpu[0].abs()
    p.K[:, :, :70, 0] = -float("inf")
    p.valid[:, :70] = False
    out, lse = p.forward()
    q, k, v, _ = p.cpu
    ref = O.Cross(q, k, v, p.valid, BF)
    near(out, ref.O, ref.O_err, "O")
    p.K[0, 0, :, 0] = -float("inf")
    out, lse = p.forward()
    assert out[0, 0].isnan().all()
    near(out[:, 1:], ref.O[:, 1:], ref.O_err[:, 1:], "O")


def test_gradient_against_differences():
    """sum(O dO) along directions of Q, K and V by central differences of the forward kernel in fp16: each value of O is
    off by half a step and P's rounding, and the step's third-order part is the cube of its size."""
    p = Problem(1, 2, 1, 20, 30, 64, FP)
    out, lse = p.forward()
    grads = p.backward(out, lse)
    g = torch.Generator().manual_seed(5)
    for name, grad in zip("QKV", grads):
        x = getattr(p, name)
        u = torch.randn(x.shape, generator=g).cuda()
        u /= u.square().mean().sqrt()
        h, loss, at, size = 0.06, [], [], 0.0
        for s in (1.0, -1.0):
            setattr(p, name, (x + s * h * u).to(FP))
            at.append(getattr(p, name).double())
            o = p.forward()[0].double()
            loss.append((o * p.dO.double()).sum())
            size = max(size, float((o * p.dO.double()).abs().sum()))
        setattr(p, name, x)
        got, want = float((grad.double() * (at[0] - at[1])).sum()), float(loss[0] - loss[1])
        # scores move by up to h |k| ~ 0.06 * 1.2 * 4 sigma: a third-order part of (0.3)^3 / 6 of the size
        assert abs(got - want) <= size * (4 * 2.0 ** -11 + 0.3 ** 3 / 6), (name, got, want, size)


def test_streams_and_graph():
    p = Problem(2, 4, 2, 300, 200, mask="mask")
    out, lse = p.forward()
    grads = p.backward(out, lse)
    want = [t.clone() for t in [out, lse] + grads]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = p.forward()
    assert torch.equal(a[0], want[0])
    b = p.backward(*p.forward(stream=s), stream=s)
    assert all(torch.equal(x, y) for x, y in zip(b, want[2:]))
    other = Problem(1, 2, 2, 900, 700)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.op.forward(p.Q, p.K, p.V, out, lse, **p.kw)
        p.op.backward(p.Q, p.K, p.V, out, lse, p.dO, *grads, **p.kw)
    for _ in range(3):
        for t in [out, lse] + grads:
            t.zero_()
        other.backward(*other.forward())
        torch.cuda.synchronize()
        g.replay()
        other.backward(*other.forward())
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip([out, lse] + grads, want))


def test_wrong_tensors_refused():
    p = Problem(1, 4, 2, 33, 20)
    out = torch.empty((1, 4, 33, 128), dtype=BF, device="cuda")
    for q in (p.Q.cpu(), p.Q.half(), p.Q[:, :3], p.Q[:, :, :, :64], p.Q.transpose(2, 3).contiguous().transpose(2, 3)):
        with pytest.raises(vc.VcError):
            p.op.forward(q, p.K, p.V, out)
    with pytest.raises(vc.VcError):
        p.op.forward(p.Q, p.K, p.V, out, k_len=torch.ones(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(vc.VcError):
        p.op.forward(p.Q, p.K, p.V, out, k_mask=torch.ones((1, 20), dtype=torch.uint8, device="cuda"))   # not masked
    with pytest.raises(vc.VcError):
        p.op.forward(p.Q, p.K, p.V, out[:, :, :1].expand(1, 4, 33, 128))
    op = vc.CrossAttention(1, 4, 2, 33, 20, masked=True)
    with pytest.raises(vc.VcError):
        op.forward(p.Q, p.K, p.V, out)   # masked, without a mask


@pytest.mark.parametrize("H,M", [(2, 40), (256, 300)])
@pytest.mark.parametrize("N,shared", [(1, False), (70, True)])
def test_infinite_value_of_few_or_shared_keys(H, M, N, shared):
    # one key, or one row for all keys (stride 0): nothing behind the last key is taken for another
    p = Problem(1, H, H, M, N)
    p.V[:, :, 0, 9] = float("inf")
    if shared:
        p.V = p.V[:, :, :1].expand(1, H, N, 128)
    out, _ = p.forward()
    assert (out[..., 9] == float("inf")).all()
    keep = torch.arange(128, device="cuda") != 9
    assert out[..., keep].isfinite().all()
    if shared or N == 1:   # every value is the one row: O is off by the roundings of P (half a step) and of O
        v = p.V[:, :, :1, keep].double()
        assert ((out[..., keep].double() - v).abs() <= 2.02 * 2.0 ** -8 * v.abs()).all()


def test_small_probabilities_in_fp16():
    """4095 keys at 2^-23.6 of one key with values of 0: their share of O is in probabilities far below fp16's normal range
    of numbers up to 1. Scores are exact (one product); a probability is rounded in steps of 2^-31 of the largest or finer."""
    N, d = 4096, 64
    for H, M in ((1, 40), (256, 260)):
        q = torch.zeros((1, H, M, d), dtype=FP, device="cuda")
        k = torch.zeros((1, H, N, d), dtype=FP, device="cuda")
        v = torch.ones_like(k)
        q[..., 0], k[:, :, 1:, 0], v[:, :, 0] = 1.0, -23.6, 0.0
        o = torch.empty_like(q)
        vc.CrossAttention(1, H, H, M, N, d, dtype=FP, sm_scale=0.6931471805599453).forward(q, k, v, o)
        x = float(k[0, 0, 1, 0].double())
        small = 2.0 ** x
        want = 4095 * small / (1 + 4095 * small)
        # scale * log2(e) is 1 within 2^-23, times 23.6: a relative error of 2^-18; fp32 sums of 4096 terms: 2^-12
        err = 2.0 ** -11 * want + 4095 * 2.0 ** -32 + (2.0 ** -18 + 2.0 ** -12) * want
        assert float((o.double() - want).abs().max()) <= err


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,H,M,N,d", [(1, 2, 150, 200, 128), (2, 2, 40, 77, 64), (1, 1, 16, 2500, 128)])
def test_keys_with_a_common_part(dtype, B, H, M, N, d):
    """Keys of large channel means, which the dS of a row cancel. dQ is rounded by at most half a step, so that this alone
    leaves an rms error of half a step of its rms; a tenth of that is left for the sums in fp32. (Roundings of dS, 0.4 of half a
    step in rms, times means of 8 times the keys' spread would leave 3.5 of it.)"""
    p = Problem(B, H, H, M, N, d, dtype, gain=0.2)
    shift = (10.0 * torch.randn((1, H, 1, d), generator=torch.Generator().manual_seed(9))).to(dtype)
    p.cpu[1] = p.cpu[1] + shift
    p.K = p.cpu[1].cuda()
    q, k, v, do = p.cpu
    ref = O.Cross(q, k, v, p.valid, dtype, 0.0, do)
    dQ = p.backward(*p.forward())[0].cpu().double()
    near(dQ, ref.dQ, ref.dQ_err, "dQ")
    rms = lambda t: float(t.square().mean().sqrt())  # noqa: E731
    assert rms(dQ - ref.dQ) <= 1.1 * O.HALF[dtype] * rms(ref.dQ)


@pytest.mark.parametrize("M", [40, 300])
def test_gradients_of_many_keys_in_fp16(M):
    # probabilities of 1 / 20000, below fp16's normal numbers
    p = Problem(1, 1, 1, M, 20000, 64, FP, gain=0.3)
    q, k, v, do = p.cpu
    ref = O.Cross(q, k, v, p.valid, FP, 0.0, do)
    dV = p.backward(*p.forward())[2]
    near(dV, ref.dV, ref.dV_fine, "dV")
    small = ref.dV.abs().square().mean().sqrt()
    assert float((dV.cpu().double() - ref.dV).square().mean().sqrt() / small) < 2.0 ** -11   # two roundings' rms is 0.7 of it


@pytest.mark.parametrize("M,scale", [(150, 0.0), (40, 40.0)])
def test_one_key_has_no_gradient_of_scores(M, scale):
    """dS of a single key is 0: what is left of dP is its fp32 sums' roundings (d + 8 of 2^-24 of its terms' sizes), not the
    error of lse (2^-24 of the scores, of several thousand), which P and with it delta's terms carry"""
    p = Problem(1, 2, 2, M, 1, scale=scale, gain=10.0)
    dQ, dK, _ = (t.cpu().double() for t in p.backward(*p.forward()))
    q, k, v, do = (t.double() for t in p.cpu)
    left = 136 * 2.0 ** -24 * (do.abs() @ v.abs().transpose(2, 3)) * (scale or 128 ** -0.5)
    assert (dQ.abs() <= left * k.abs()).all()
    assert (dK.abs() <= (left * q.abs()).sum(2, keepdim=True)).all()


@pytest.mark.parametrize("N", [1023, 4096, 4097, 16400, 40001])
def test_lists_of_many_keys(N):
    """masks of more keys than a pass over them takes, rows of the mask at odd addresses, an item of which no key counts and
    one of which all do: O of the masked keys is that of the keys that are left, to the order of the sums"""
    g = torch.Generator().manual_seed(N)
    rand = lambda *s: torch.randn(s, generator=g).to(BF).cuda()  # noqa: E731
    B, H, M, d = 4, 1, 3, 64
    Q, K, V = rand(B, H, M, d), rand(B, H, N, d), rand(B, H, N, d)
    mask = (torch.rand((B, N), generator=g) < 0.5)
    mask[1], mask[2] = True, False
    wide = torch.zeros((B, N + 3), dtype=torch.bool, device="cuda")
    wide[:, 1:N + 1] = mask.cuda()
    k_len = torch.tensor([N, N, N, N // 2], dtype=torch.int32)
    out, lse = torch.empty_like(Q), torch.empty((B, H, M), device="cuda")
    vc.CrossAttention(B, H, H, M, N, d, masked=True).forward(Q, K, V, out, lse, k_len=k_len.cuda(), k_mask=wide[:, 1:N + 1])
    mask &= torch.arange(N)[None] < k_len[:, None]
    ref = O.Cross(Q.cpu(), K.cpu(), V.cpu(), mask, BF)
    near(out, ref.O, ref.O_err, "O")
    assert (out[2] == 0).all() and (lse[2] == -float("inf")).all()
    keep = torch.tensor([0, 1, 3])
    assert ((lse.cpu().double() - ref.lse)[keep].abs() <= ref.lse_err[keep].expand(3, H, M)).all()
