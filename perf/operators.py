"""Timed cases of the operators that stand around the attention of a transformer block.

  xattn   attention of queries to the states of another sequence (an encoder's), of another length:
          O = softmax(scale Q K^T) V with grouped key heads, key lengths and key padding masks;
          `train` also forms dQ, dK and dV of a given dO
  nr      RMS norms of queries and keys (of each head, or over all heads of a token) and the rotation
          by position in the same pass, from the packed projection; `train` also forms the gradients of
          the inputs and of the norms' weights
  rot     that rotation alone: interleaved or half layout, the whole head or a part of it, angles scaled
          for long contexts; `train` also forms the gradients

With `own` false everything is elementary torch in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
THETA = 10000.0
EPS = 1e-6

MOST_FLOPS = 4.0 * 40 * 75600 * 512 * 128   # the forward attention of the largest listed case
MOST_ROWS = 40 * 75600                      # rows of one of its tensors
MOST_NR_ROWS = 2 * 12 * 32760               # rows of queries and keys of the largest listed norm


def _xattn(train, B, Hq, Hk, M, N, d=128, dtype="bf16", mask="none", packed=True, name=None):
    c = dict(op="xattn", train=train, B=B, Hq=Hq, Hk=Hk, M=M, N=N, d=d, dtype=dtype, mask=mask, packed=packed)
    return dict(c, name=name) if name else c


def _nr(op, train, B, Hq, Hk, grid, N=0, d=128, dtype="bf16", norm="head", layout="interleaved", rot=128, stretch=1.0,
        far=0, name=None):
    F, Ht, Wd = grid
    c = dict(op=op, train=train, B=B, Hq=Hq, Hk=Hk, F=F, Ht=Ht, Wd=Wd, N=N or F * Ht * Wd, d=d, dtype=dtype, norm=norm,
             layout=layout, rot=rot, stretch=stretch, far=far)
    return dict(c, name=name) if name else c


LINE = (0, 0, 0)   # positions on a line instead of a latent grid


def listed():
    return [
        # one new token of a decoder that attends to 1500 encoder states, four query heads to a key head:
        # the smallest call, latency
        _xattn(False, 1, 32, 8, 1, 1500, name="xattn_token_gqa"),
        # the smallest layer's 1024 tokens against a short odd prompt, fp16
        _xattn(False, 1, 2, 2, 1024, 77, dtype="fp16", packed=False, name="xattn_1024_h2_n77_fp16"),
        # the 12-head layer of 32760 tokens against 512 encoder states: the ordinary call
        _xattn(False, 1, 12, 12, 32760, 512, name="xattn_32760_h12"),
        # the 40-head layer of 75600 tokens: the largest call
        _xattn(False, 1, 40, 40, 75600, 512, name="xattn_75600_h40"),
        # 64 learned queries that pool the states of 32760 tokens
        _xattn(False, 1, 12, 12, 64, 32760, name="xattn_pool_64_n32760"),
        # training of the 12-head layer
        _xattn(True, 1, 12, 12, 32760, 512, name="xattn_train_32760_h12"),
        # training on a ragged padded batch, odd lengths, shared key heads of 64 channels, one item without a key
        _xattn(True, 3, 8, 2, 1021, 257, d=64, mask="mask", name="xattn_train_padded_b3_d64"),
        # one new token of each of 16 sequences far into a long context, norms per head, half layout
        _nr("nr", False, 16, 32, 8, LINE, N=1, layout="half", far=100000, name="nr_token_b16"),
        # the 12-head layer's norm over the whole token and the three-axis rotation
        _nr("nr", False, 1, 12, 12, (21, 39, 40), norm="token", name="nr_32760_h12_token"),
        # training of that layer with norms per head
        _nr("nr", True, 1, 12, 12, (21, 39, 40), name="nr_train_32760_h12"),
        # the rotation alone of a long prompt: half layout, half of the head, angles stretched eightfold, fp16
        _nr("rot", False, 1, 32, 8, LINE, N=16381, dtype="fp16", norm="none", layout="half", rot=64, stretch=8.0,
            name="rot_16381_part_fp16"),
        # training of a small batch, interleaved layout
        _nr("rot", True, 2, 7, 7, LINE, N=1000, norm="none", name="rot_train_1000_b2"),
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    op = rng.choice(["xattn", "xattn", "nr", "rot"])
    train = rng.random() < 0.4
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    d = rng.choice([128, 128, 64])
    if op == "xattn":
        while True:
            shape = rng.choice(["few", "layer", "layer", "pool"])
            if shape == "few":          # some tokens of a decoder
                M, N, B = _log(rng, 1, 16), _log(rng, 1, 8192), _log(rng, 1, 32)
            elif shape == "layer":      # many tokens, a prompt
                M, N, B = _log(rng, 17, 75600), _log(rng, 1, 2048), _log(rng, 1, 4)
            else:                       # pooling of many states
                M, N, B = _log(rng, 8, 512), _log(rng, 2048, 32760), _log(rng, 1, 2)
            Hk = _log(rng, 1, 40)
            Hq = Hk * rng.choice([1, 1, 1, 2, 4, 7])
            flops = 4.0 * B * Hq * M * N * d * (3.5 if train else 1.0)
            if Hq <= 40 and flops <= MOST_FLOPS and B * Hq * M * (2 if train else 1) <= MOST_ROWS:
                break
        mask = rng.choice(["none", "none", "len", "mask"])
        return _xattn(train, B, Hq, Hk, M, N, d, dtype, mask, rng.random() < 0.6)
    while True:
        norm = "none" if op == "rot" else rng.choice(["head", "token"])
        layout = rng.choice(["interleaved", "half"])
        Hk = _log(rng, 1, 40)
        Hq = Hk * rng.choice([1, 1, 2, 4])
        grid, N, rot, far, stretch = LINE, 0, d, 0, 1.0
        if d == 128 and rng.random() < 0.5:
            n = math.exp(rng.uniform(math.log(64), math.log(75600)))
            F = rng.randint(1, min(21, max(1, int(n / 64))))
            Ht = max(1, round(math.sqrt(n / F) * math.exp(rng.uniform(-0.5, 0.3))))
            grid = (F, Ht, max(1, round(n / F / Ht)))
            B, N = rng.choice([1, 1, 2]), grid[0] * grid[1] * grid[2]
        else:
            B, N = _log(rng, 1, 16), _log(rng, 1, 32760)
            rot = rng.choice([d, d, d // 2, 16, d - 16])
            far = rng.choice([0, 0, 100000])
            stretch = rng.choice([1.0, 1.0, 4.0, 8.0])
        if Hq <= 40 and B * (Hq + Hk) * N * (2 if train else 1) <= MOST_NR_ROWS * (2 if train else 1):
            break
    return _nr(op, train, B, Hq, Hk, grid, N, d, dtype, norm, layout, rot, stretch, far)


# ---- inputs ----------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 5 + 3)
    return dict(device="cuda", generator=g)


def _tokens(e, B, n, H, d, dtype, gain=1.0, offset=0.0):
    """[B, n, H, d]: tokens with a gain and channel offsets of each head, and two outlier channels."""
    x = torch.randn((B, n, H, d), **e)
    g = gain * torch.exp(0.3 * torch.randn((H, 1), **e)).expand(H, d).clone()
    g.scatter_(1, torch.rand((H, d), **e).topk(2, 1).indices, 2.0 * gain)
    x.mul_(g).add_(offset * torch.randn((H, d), **e))
    return x.to(TYPES[dtype])


def _valid(c):
    """Valid keys of each item of a padded batch: from all of them to none at the last."""
    if c["mask"] == "none":
        return [c["N"]] * c["B"]
    if c["B"] == 1:
        return [c["N"] - c["N"] // 3]
    return [c["N"] * (c["B"] - 1 - b) // (c["B"] - 1) for b in range(c["B"])]


def _prepare_xattn(c, seed):
    e = _gen(seed)
    B, Hq, Hk, M, N, d, dt = c["B"], c["Hq"], c["Hk"], c["M"], c["N"], c["d"], c["dtype"]
    q = _tokens(e, B, M, Hq, d, dt, gain=1.3)
    kv = torch.stack([_tokens(e, B, N, Hk, d, dt, gain=1.2, offset=0.5), _tokens(e, B, N, Hk, d, dt, offset=0.5)], 2)
    heads = lambda t: t.transpose(1, 2)  # noqa: E731
    Q, K, V = heads(q), heads(kv[:, :, 0]), heads(kv[:, :, 1])
    if not c["packed"]:
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
    s = dict(Q=Q, K=K, V=V, k_len=None, k_mask=None)
    valid = torch.tensor(_valid(c), dtype=torch.int32, device="cuda")
    if c["mask"] == "len":
        s["k_len"] = valid
    elif c["mask"] == "mask":
        rank = torch.rand((B, N), **e).argsort(1).argsort(1)
        s["k_mask"] = (rank < valid[:, None]).to(torch.uint8)
    if c["train"]:
        s["dO"] = heads(_tokens(e, B, M, Hq, d, dt))
    if own:
        import paper_2609_15810_amd as vc
        s["op"] = vc.CrossAttention(B, Hq, Hk, M, N, d, dtype=TYPES[dt], masked=c["mask"] == "mask",
                                    training=c["train"])
        s["O"] = torch.empty_like(Q)
        if c["train"]:
            s["lse"] = torch.empty((B, Hq, M), dtype=torch.float32, device="cuda")
            s["dQ"], s["dK"], s["dV"] = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
    return s


def _frequencies(c, dtype, device="cuda"):
    """Angles per position of the rotated pairs of a line: the base's, and with `stretch` the interpolation
    by parts: pairs that turn more than 32 times over the 4096 positions of the training stay as they are, pairs
    that turn less than once are slowed by the factor, those between mixed."""
    half = c["rot"] // 2
    f = THETA ** (-torch.arange(half, dtype=dtype, device=device) / half)
    if c["stretch"] > 1.0:
        turns = 4096.0 * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
        f = f * keep + f / c["stretch"] * (1.0 - keep)
    return f


def _tables(c):
    """cos and sin tables in fp32, formed in 64 bits: of a grid one row per frame, row and column, pairs 0..21
    turning with the frame, 22..42 with the row and 43..63 with the column; of a line one row per position."""
    if c["F"]:
        rows = []
        for axis, n in enumerate((c["F"], c["Ht"], c["Wd"])):
            first, pairs = (0, 22, 43)[axis], (22, 21, 21)[axis]
            ang = torch.zeros((n, 64), dtype=torch.float64, device="cuda")
            j = torch.arange(pairs, dtype=torch.float64, device="cuda")
            ang[:, first:first + pairs] = torch.arange(n, device="cuda")[:, None] * THETA ** (-j / pairs)
            rows.append(ang)
        ang, scale = torch.cat(rows), 1.0
    else:
        n = c["far"] + c["N"]
        ang = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * _frequencies(c, torch.float64)
        scale = 0.1 * math.log(c["stretch"]) + 1.0
    return (ang.cos() * scale).float().contiguous(), (ang.sin() * scale).float().contiguous()


def _prepare_nr(c, seed):
    e = _gen(seed)
    B, Hq, Hk, N, d, dt = c["B"], c["Hq"], c["Hk"], c["N"], c["d"], c["dtype"]
    qkv = _tokens(e, B, N, Hq + 2 * Hk, d, dt, gain=2.0, offset=0.5)
    heads = lambda t: t.transpose(1, 2)  # noqa: E731
    s = dict(q=heads(qkv[:, :, :Hq]), k=heads(qkv[:, :, Hq:Hq + Hk]), pos=None, q_weight=None, k_weight=None)
    s["cos"], s["sin"] = _tables(c)
    if c["far"]:
        # every sequence at its own place
        start = torch.randint(0, c["far"], (B, 1), **e)
        s["pos"] = (start + torch.arange(N, device="cuda")).to(torch.int32)
    if c["norm"] != "none":
        span = (lambda H: d) if c["norm"] == "head" else (lambda H: H * d)
        s["q_weight"] = 1.0 + 0.2 * torch.randn(span(Hq), **e)
        s["k_weight"] = 1.0 + 0.2 * torch.randn(span(Hk), **e)
    if c["train"]:
        s["dq_out"] = heads(_tokens(e, B, N, Hq, d, dt)).contiguous()
        s["dk_out"] = heads(_tokens(e, B, N, Hk, d, dt)).contiguous()
    if own:
        import paper_2609_15810_amd as vc
        s["op"] = vc.NormRope(B, Hq, Hk, N, d, dtype=TYPES[dt],
                              norm=dict(none=vc.NORM_NONE, head=vc.NORM_HEAD, token=vc.NORM_TOKEN)[c["norm"]], eps=EPS,
                              layout=dict(interleaved=vc.ROPE_INTERLEAVED, half=vc.ROPE_HALF)[c["layout"]],
                              rot=c["rot"], grid=(c["F"], c["Ht"], c["Wd"]) if c["F"] else None, training=c["train"])
        new = lambda H: torch.empty((B, H, N, d), dtype=TYPES[dt], device="cuda")  # noqa: E731
        s["q_out"], s["k_out"] = new(Hq), new(Hk)
        if c["train"]:
            dqkv = torch.empty_like(qkv)
            s["dq"], s["dk"] = heads(dqkv[:, :, :Hq]), heads(dqkv[:, :, Hq:Hq + Hk])
            for w in ("q_weight", "k_weight"):
                s["d" + w] = None if s[w] is None else torch.empty_like(s[w])
    return s


def prepare(case, seed):
    s = _prepare_xattn(case, seed) if case["op"] == "xattn" else _prepare_nr(case, seed)
    return dict(s, case=dict(case))


# ---- the plain forms ---------------------------------------------------------------------------------

def _plain_xattn(s, c):
    B, Hq, Hk, M, N, d = (c[k] for k in ("B", "Hq", "Hk", "M", "N", "d"))
    dt = TYPES[c["dtype"]]
    rows = Hq // Hk * M   # the query heads of a key head, one behind the other
    scale = 1.0 / math.sqrt(d)
    q = s["Q"].float().reshape(B, Hk, rows, d)
    k, v = s["K"].float(), s["V"].float()
    out = None
    if c["mask"] != "none":
        j = torch.arange(N, device="cuda")
        out = (j >= s["k_len"][:, None]) if c["mask"] == "len" else s["k_mask"] == 0
        out = out[:, None, None, :]
    x = torch.matmul(q, k.transpose(2, 3)).mul_(scale)
    if out is not None:
        x.masked_fill_(out, -math.inf)
    top = x.amax(3, keepdim=True)
    if out is not None:
        top = top.masked_fill(top == -math.inf, 0.0)
    p = x.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    if out is not None:
        total = total.masked_fill(total == 0.0, 1.0)
    p.div_(total)
    o = torch.matmul(p, v)
    res = dict(O=o.reshape(B, Hq, M, d).to(dt))
    if c["train"]:
        do = s["dO"].float().reshape(B, Hk, rows, d)
        res["dV"] = torch.matmul(p.transpose(2, 3), do).to(dt)
        dp = torch.matmul(do, v.transpose(2, 3))
        ds = dp.sub_((do * o).sum(3, keepdim=True)).mul_(p).mul_(scale)
        res["dQ"] = torch.matmul(ds, k).reshape(B, Hq, M, d).to(dt)
        res["dK"] = torch.matmul(ds.transpose(2, 3), q).to(dt)
    return res


def _angles(s, c):
    """cos and sin [B or 1, N, rot / 2] of the tokens' pairs."""
    if c["F"]:
        F, Ht, Wd = c["F"], c["Ht"], c["Wd"]
        n = torch.arange(c["N"], device="cuda")
        idx = (n // (Ht * Wd), F + n // Wd % Ht, F + Ht + n % Wd)
        pick = lambda t: torch.cat([t[i][:, a:b] for i, (a, b) in zip(idx, ((0, 22), (22, 43), (43, 64)))], 1)  # noqa: E731
        return pick(s["cos"])[None], pick(s["sin"])[None]
    if s["pos"] is None:
        return s["cos"][None, :c["N"]], s["sin"][None, :c["N"]]
    pos = s["pos"].long()
    return s["cos"][pos], s["sin"][pos]


def _turn(x, cos, sin, c):
    """Rotate the first rot channels of x [B, H, N, d]."""
    rot = c["rot"]
    cos, sin = cos[:, None], sin[:, None]
    y = x.clone()
    if c["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, a * sin + b * cos
    return y


def _plain_nr(s, c):
    dt = TYPES[c["dtype"]]
    cos, sin = _angles(s, c)
    dims = (1, 3) if c["norm"] == "token" else 3
    res = {}
    for t in ("q", "k"):
        x, w = s[t].float(), s[t + "_weight"]
        if c["norm"] == "none":
            res[t + "_out"] = _turn(x, cos, sin, c).to(dt)
            if c["train"]:
                res["d" + t] = _turn(s["d%s_out" % t].float(), cos, -sin, c).to(dt)
            continue
        if c["norm"] == "token":
            w = w.view(x.shape[1], 1, x.shape[3])
        r = torch.rsqrt((x * x).mean(dims, keepdim=True) + EPS)
        xr = x * r
        res[t + "_out"] = _turn(xr * w, cos, sin, c).to(dt)
        if c["train"]:
            g = _turn(s["d%s_out" % t].float(), cos, -sin, c)
            dw = (g * xr).sum((0, 2))
            res["d%s_weight" % t] = dw.reshape(-1) if c["norm"] == "token" else dw.sum(0)
            g = g * w
            res["d" + t] = (r * (g - xr * (g * xr).mean(dims, keepdim=True))).to(dt)
    return res


# ---- the timed pass ------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if not own:
        return _plain_xattn(s, c) if c["op"] == "xattn" else _plain_nr(s, c)
    op = s["op"]
    if c["op"] == "xattn":
        m = dict(k_len=s["k_len"], k_mask=s["k_mask"])
        if not c["train"]:
            op.forward(s["Q"], s["K"], s["V"], s["O"], **m)
            return dict(O=s["O"])
        op.forward(s["Q"], s["K"], s["V"], s["O"], s["lse"], **m)
        op.backward(s["Q"], s["K"], s["V"], s["O"], s["lse"], s["dO"], s["dQ"], s["dK"], s["dV"], **m)
        return {k: s[k] for k in ("O", "dQ", "dK", "dV")}
    w = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], cos=s["cos"], sin=s["sin"], pos=s["pos"])
    op.forward(s["q"], s["k"], s["q_out"], s["k_out"], **w)
    out = {k: s[k] for k in ("q_out", "k_out")}
    if c["train"]:
        if c["norm"] == "none":
            op.backward(s["q"], s["k"], s["dq_out"], s["dk_out"], s["dq"], s["dk"], **w)
        else:
            op.backward(s["q"], s["k"], s["dq_out"], s["dk_out"], s["dq"], s["dk"], dq_weight=s["dq_weight"],
                        dk_weight=s["dk_weight"], **w)
            out.update(dq_weight=s["dq_weight"], dk_weight=s["dk_weight"])
        out.update(dq=s["dq"], dk=s["dk"])
    return out


def work(case):
    """Each input read once, each result written once; the products of the valid keys."""
    c = case
    if c["op"] == "xattn":
        rows, keys = c["B"] * c["Hq"] * c["M"], c["Hk"] * sum(_valid(c))
        pairs = c["Hq"] * c["M"] * sum(_valid(c))
        size = 2.0 * c["d"]
        if c["train"]:   # Q, dO in, O, dQ out; K, V in, dK, dV out
            return dict(bytes=size * (4 * rows + 2 * keys + 2 * c["B"] * c["Hk"] * c["N"]), flops=14.0 * pairs * c["d"])
        return dict(bytes=size * (2 * rows + 2 * keys), flops=4.0 * pairs * c["d"])
    values = c["B"] * (c["Hq"] + c["Hk"]) * c["N"] * c["d"]
    table = 4.0 * c["rot"] * ((c["F"] + c["Ht"] + c["Wd"]) if c["F"] else c["N"] * (c["B"] if c["far"] else 1))
    tensors, ops = (2, 7.0) if not c["train"] else ((4, 20.0) if c["norm"] != "none" else (4, 6.0))
    if c["norm"] == "none" and not c["train"]:
        ops = 3.0
    return dict(bytes=2.0 * tensors * values + table, flops=ops * values)


# ---- 64-bit references ------------------------------------------------------------------------------------

def _exact_xattn(s, c):
    B, Hq, Hk, M, N, d = (c[k] for k in ("B", "Hq", "Hk", "M", "N", "d"))
    new = lambda H, n: torch.zeros((B, H, n, d), dtype=torch.float64, device="cuda")  # noqa: E731
    res = dict(O=new(Hq, M))
    if c["train"]:
        res.update(dQ=new(Hq, M), dK=new(Hk, N), dV=new(Hk, N))
    step = max(1, (1 << 27) // N)
    for b in range(B):
        keys = torch.arange(N, device="cuda")
        if c["mask"] == "len":
            keys = keys[:int(s["k_len"][b])]
        elif c["mask"] == "mask":
            keys = s["k_mask"][b].nonzero()[:, 0]
        if not len(keys):
            continue
        for h in range(Hq):
            g = h * Hk // Hq
            K, V = s["K"][b, g, keys].double(), s["V"][b, g, keys].double()
            for m in range(0, M, step):
                Q = s["Q"][b, h, m:m + step].double()
                P = torch.softmax((Q @ K.T) / math.sqrt(d), 1)
                O = P @ V
                res["O"][b, h, m:m + step] = O
                if c["train"]:
                    G = s["dO"][b, h, m:m + step].double()
                    S = P * (G @ V.T - (G * O).sum(1, keepdim=True)) / math.sqrt(d)
                    res["dQ"][b, h, m:m + step] = S @ K
                    res["dK"][b, g].index_add_(0, keys, S.T @ Q)
                    res["dV"][b, g].index_add_(0, keys, P.T @ G)
    return res


def _exact_nr(s, c):
    B, N, d, rot = c["B"], c["N"], c["d"], c["rot"]
    n = torch.arange(N, device="cuda")
    if c["F"]:
        axes = (n // (c["Ht"] * c["Wd"]), n // c["Wd"] % c["Ht"], n % c["Wd"])
        ang = [p[:, None].double() * THETA ** (-torch.arange(m, dtype=torch.float64, device="cuda") / m)
               for p, m in zip(axes, (22, 21, 21))]
        ang = torch.cat(ang, 1)[None]
        scale = 1.0
    else:
        pos = n[None] if s["pos"] is None else s["pos"].long()
        ang = pos[..., None].double() * _frequencies(c, torch.float64)
        scale = 0.1 * math.log(c["stretch"]) + 1.0
    turn = torch.polar(torch.full_like(ang, scale), ang)[:, None]   # [B or 1, 1, N, rot / 2]

    def rotate(x, w):
        head = x[..., :rot]
        if c["layout"] == "half":
            z = torch.complex(head[..., :rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * w
            head = torch.cat([z.real, z.imag], -1)
        else:
            z = torch.view_as_complex(head.reshape(head.shape[:-1] + (rot // 2, 2)).contiguous()) * w
            head = torch.view_as_real(z).reshape(head.shape)
        return torch.cat([head, x[..., rot:]], -1)

    res = {}
    for t in ("q", "k"):
        x = s[t].double()
        if c["norm"] == "none":
            res[t + "_out"] = rotate(x, turn)
            if c["train"]:
                res["d" + t] = rotate(s["d%s_out" % t].double(), turn.conj())
            continue
        w = s[t + "_weight"].double()
        over = (3,)
        if c["norm"] == "token":
            w, over = w.view(1, -1, 1, d), (1, 3)
        rms = (x.square().mean(over, keepdim=True) + EPS).sqrt()
        unit = x / rms
        res[t + "_out"] = rotate(unit * w, turn)
        if c["train"]:
            g = rotate(s["d%s_out" % t].double(), turn.conj())
            dw = (g * unit).sum(0).sum(1)
            res["d%s_weight" % t] = dw.reshape(-1) if c["norm"] == "token" else dw.sum(0)
            gw = g * w
            res["d" + t] = (gw - unit * (gw * unit).mean(over, keepdim=True)) / rms
    return res


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_xattn(s, case) if case["op"] == "xattn" else _exact_nr(s, case)
