"""The operators of a block together, as they are used: the packed projection's queries and keys normed and turned
(vc_norm_rope), low-bit self attention on them (group, prep without its own rotation, forward), the queries of the attention
to a prompt normed (vc_norm_rope without rotation) and that attention (vc_cross_attn), and its gradients.

Each step is checked on what the step before left on the GPU: the norms and the attention to the prompt within the bounds of
block_oracle, the low-bit attention within rel-L2 5e-3 of the CPU oracle's identically quantized pipeline.
"""
import numpy as np
import pytest

import oracle
import synthetic as S

torch = pytest.importorskip("torch")
vc = pytest.importorskip("paper_2609_15810_amd")
import block_oracle as O  # noqa: E402

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
GRID, H, D, EPS = (4, 8, 16), 3, 128, 1e-6
N, TEXT = 4 * 8 * 16, 77


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    vc.lib()


class Block:
    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g)  # noqa: E731
        new = lambda *s: torch.empty(s, dtype=BF, device="cuda")  # noqa: E731
        self.qkv = (2.0 * rand(1, N, 3 * H, D)).to(BF).cuda()
        self.text = rand(1, TEXT, 2 * H, D).to(BF).cuda()
        self.mask = (torch.rand((1, TEXT), generator=g) < 0.7).cuda()
        self.w = [(1.0 + 0.2 * rand(H * D)).cuda() for _ in range(2)]
        self.wc = (1.0 + 0.2 * rand(D)).cuda()
        self.grad = rand(1, H, N, D).to(BF).cuda()
        self.norm = vc.NormRope(1, H, H, N, norm=vc.NORM_TOKEN, eps=EPS, grid=GRID)
        self.attn = vc.Attention(1, H, GRID, vc.make_opts(rope=False), vc.make_group_opts(k=16, iters=4))
        self.norm_c = vc.NormRope(1, H, 0, N, norm=vc.NORM_HEAD, eps=EPS, layout=vc.ROPE_NONE)
        self.cross = vc.CrossAttention(1, H, H, N, TEXT, masked=True, training=True)
        self.q, self.k, self.v, self.o, self.qc, self.oc, self.dqc = (new(1, H, N, D) for _ in range(7))
        self.lse = torch.empty((1, H, N), device="cuda")
        self.dtext = torch.empty_like(self.text)

    def heads(self, packed):
        t = packed.transpose(1, 2)
        return [t[:, i * H:(i + 1) * H] for i in range(t.shape[1] // H)]

    def run(self):
        q, k, v = self.heads(self.qkv)
        self.norm.forward(q, k, self.q, self.k, *self.w, self.attn.rope_cos, self.attn.rope_sin)
        self.v.copy_(v)
        self.attn.group(self.v)
        self.attn.prep(self.q, self.k, self.v)
        self.attn.forward(self.o)
        self.norm_c.forward(self.o, None, self.qc, None, q_weight=self.wc)
        K, V = self.heads(self.text)
        self.cross.forward(self.qc, K, V, self.oc, self.lse, k_mask=self.mask)
        self.cross.backward(self.qc, K, V, self.oc, self.lse, self.grad, self.dqc, *self.heads(self.dtext),
                            k_mask=self.mask)

    def results(self):
        return [self.q, self.k, self.o, self.qc, self.oc, self.lse, self.dqc, self.dtext]


def close(got, ref, err):
    assert ((got.cpu().double() - ref).abs() <= err).all()


def test_block():
    b = Block(1)
    b.run()
    torch.cuda.synchronize()
    # norms and rotation
    half = O.HALF[BF]
    ang = O.grid_angles(*GRID)[None]
    for x, w, got in zip(b.heads(b.qkv), b.w, (b.q, b.k)):
        x, w = x.cpu().double(), w.cpu().double()
        ref = O.norm_rope(x, w, ang.cos(), ang.sin(), "interleaved", D, "token", EPS)
        size = O.pair_size(O.norm_rope(x, w, ang.cos(), ang.sin(), "none", 0, "token", EPS), "interleaved", D)
        close(got, ref, half * (ref.abs() + 2.0 ** -17 * size) + 2.0 ** -17 * size)   # see test_gpu_norm_rope.py
    # low-bit attention
    bits = lambda t: np.ascontiguousarray(t.cpu().view(torch.int16).numpy()).view(np.uint16)  # noqa: E731
    g = oracle.group(bits(b.v), GRID, k=16, iters=4)
    assert np.array_equal(b.attn.perm.cpu().numpy(), g["perm"])
    pp = oracle.prep(bits(b.q), bits(b.k), bits(b.v), GRID, perm=g["perm"], rope=False)
    ref = oracle.attention(pp, np.arange(N))
    o = S.bits_to_f32(bits(b.o)).reshape(H, N, D).astype(np.float64)
    assert np.linalg.norm(o - ref) <= 5e-3 * np.linalg.norm(ref)
    # the queries of the attention to the prompt, and that attention
    c = s = torch.zeros((1, N, 1), dtype=torch.float64)
    x = b.o.cpu().double()
    ref = O.norm_rope(x, b.wc.cpu().double(), c, s, "none", 0, "head", EPS)
    close(b.qc, ref, half * ref.abs() * (1 + 2.0 ** -16) + 2.0 ** -17 * ref.abs())
    K, V = (t.cpu() for t in b.heads(b.text))
    r = O.Cross(b.qc.cpu(), K, V, b.mask.cpu(), BF, dO=b.grad.cpu())
    dK, dV = b.heads(b.dtext)
    for got, name in ((b.oc, "O"), (b.dqc, "dQ"), (dK, "dK"), (dV, "dV")):
        close(got, getattr(r, name), getattr(r, name + "_err"))


def test_block_captured():
    b, other = Block(2), Block(3)
    b.run()
    want = [t.clone() for t in b.results()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run()
    for _ in range(3):
        for t in b.results():
            t.zero_()
        other.run()
        torch.cuda.synchronize()
        graph.replay()
        other.run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(b.results(), want))


def test_two_streams_at_once():
    blocks = [Block(4), Block(5)]
    want = []
    for b in blocks:
        b.run()
        want.append([t.clone() for t in b.results()])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                b.run()
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        assert all(torch.equal(x, y) for x, y in zip(b.results(), w))
