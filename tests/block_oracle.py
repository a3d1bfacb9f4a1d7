"""Plain 64-bit forms of the operators around the attention (test infrastructure: torch on the CPU)."""
import math

import torch

# half a step of a type, relative to the value, and half its smallest step
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def angles(pos, rot, theta=10000.0):
    """[.., rot/2] angles of positions on a line"""
    i = torch.arange(rot // 2, dtype=torch.float64)
    return pos.double()[..., None] * theta ** (-2.0 * i / rot)


def grid_angles(F, Ht, Wd, theta=10000.0):
    """[N, 64]: pairs 0..21 turn with the frame, 22..42 with the row, 43..63 with the column"""
    n = torch.arange(F * Ht * Wd)
    out = []
    for p, pairs in ((n // (Ht * Wd), 22), (n // Wd % Ht, 21), (n % Wd, 21)):
        out.append(p.double()[:, None] * theta ** (-torch.arange(pairs, dtype=torch.float64) / pairs))
    return torch.cat(out, 1)


def turn(x, cos, sin, layout, rot):
    """x [B, H, N, d]; cos, sin [B or 1, N, rot/2]; layout "half", "interleaved" or "none" """
    if layout == "none":
        return x
    cos, sin, y = cos[:, None], sin[:, None], x.clone()
    lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., lo] = x[..., lo] * cos - x[..., hi] * sin
    y[..., hi] = x[..., lo] * sin + x[..., hi] * cos
    return y


def norm_rope(x, w, cos, sin, layout, rot, norm, eps):
    """x [B, H, N, d] fp64, w fp64 or None; returns the output"""
    if norm != "none":
        over = (1, 3) if norm == "token" else (3,)
        x = x / (x.square().mean(over, keepdim=True) + eps).sqrt()
        if w is not None:
            x = x * (w.view(1, x.shape[1], 1, x.shape[3]) if norm == "token" else w)
    return turn(x, cos, sin, layout, rot)


def pair_size(x, layout, rot):
    """|a| + |b| of each channel's pair (|x| where it is not turned): what a rotation's fp32 errors are relative to"""
    if layout == "none":
        return x.abs()
    y = x.abs().clone()
    lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., lo] = y[..., hi] = x[..., lo].abs() + x[..., hi].abs()
    return y


def norm_rope_grad(x, w, cos, sin, layout, rot, norm, eps, dz):
    """dx, dw, and the sizes of the terms that each is a sum of"""
    g = turn(dz, cos, -sin, layout, rot)
    gs = pair_size(dz, layout, rot) * math.sqrt(float((cos ** 2 + sin ** 2).max())) if layout != "none" else dz.abs()
    if norm == "none":
        return g, None, gs, None
    over = (1, 3) if norm == "token" else (3,)
    r = 1.0 / (x.square().mean(over, keepdim=True) + eps).sqrt()
    u = x * r
    ww = torch.ones(()).double() if w is None else (w.view(1, x.shape[1], 1, x.shape[3]) if norm == "token" else w)
    dw, dws = (g * u).sum((0, 2)), (gs * u.abs()).sum((0, 2))
    if norm == "head":
        dw, dws = dw.sum(0), dws.sum(0)
    dx = r * (g * ww - u * (g * ww * u).mean(over, keepdim=True))
    dxs = r * (gs * ww.abs() + u.abs() * (gs * (ww * u).abs()).mean(over, keepdim=True))
    return dx, dw.reshape(-1), dxs, dws.reshape(-1)


class Cross:
    """Attention to another sequence and its gradients in 64 bits, with bounds of a kernel's errors.

    What a kernel may do: round P and dS to the type (half a step each), round outputs (half a step), and compute in fp32: scores of d products (d + 8 steps of 2^-24 of the
    sum of their sizes, in log2 units, which the exponential turns into a relative error, once for the score and once
    for lse), sums over the keys (at most N + 64 additions of 2^-24 each). In fp16 P and dS below the normal range
    round absolutely (TINY).
    """

    def __init__(self, Q, K, V, valid, dtype, scale=0.0, dO=None):
        half, tiny = HALF[dtype], TINY[dtype]
        Q, K, V = Q.double(), K.double(), V.double()
        B, Hq, M, d = Q.shape
        Hk, N = K.shape[1], K.shape[2]
        scale = scale or 1.0 / math.sqrt(d)
        on = valid[:, :, None].to(torch.bool)
        zero = torch.zeros((), dtype=torch.float64)
        K, V = (torch.where(on[:, None], t, zero) for t in (K, V))
        Kg, Vg = (t.repeat_interleave(Hq // Hk, 1) for t in (K, V))
        off = ~valid[:, None, None, :].to(torch.bool)
        S = (Q @ Kg.transpose(2, 3)).mul(scale).masked_fill(off, -math.inf)
        self.lse = torch.logsumexp(S, 3)
        P = torch.exp(S - torch.where(self.lse == -math.inf, zero, self.lse)[..., None])
        P = P.masked_fill(off, 0.0)
        self.O = P @ Vg
        size = float((Q.abs() @ Kg.abs().transpose(2, 3)).max()) * scale * 1.4427
        rel = 2 * 0.6932 * (d + 8) * 2.0 ** -24 * size + (N + 64) * 2.0 ** -24 + 2.0 ** -20
        A = P @ Vg.abs()
        self.O_err = half * (1 + half) * self.O.abs() + (1 + half) * (half + rel) * A + \
            tiny * (1 + Vg.abs().sum(2, keepdim=True)) * 1.01
        self.lse_err = rel + 2.0 ** -22 * torch.where(self.lse == -math.inf, zero, self.lse).abs()
        if dO is None:
            return
        G = dO.double()
        group = lambda t: t.view(B, Hk, Hq // Hk, N, d).sum(2)  # noqa: E731
        dP = G @ Vg.transpose(2, 3)
        dPs = G.abs() @ Vg.abs().transpose(2, 3)
        delta = (P * dP).sum(3, keepdim=True)
        dS = P * (dP - delta)
        derr = ((rel + d * 2.0 ** -24) * P * dPs).sum(3, keepdim=True)
        dSerr = P * ((half + rel) * (dP - delta).abs() + d * 2.0 ** -24 * dPs + derr) * (1 + half)
        Pt = P.transpose(2, 3)
        self.dV, self.dQ = group(Pt @ G), dS @ Kg * scale
        self.dK = group(dS.transpose(2, 3) @ Q) * scale
        out = lambda ref, err: half * ref.abs() + (1 + half) * err + tiny  # noqa: E731
        rows = Hq // Hk * M
        add = 1 + (rows + N) * 2.0 ** -24   # fp32 sums over rows or keys, of terms of these sizes
        self.dV_err = out(self.dV, add * group((half + rel) * Pt @ G.abs()) + (rows * 2.0 ** -24) * group(Pt @ G.abs()) +
                          tiny * group(G.abs().sum(2, keepdim=True).expand(B, Hq, N, d)))
        # as dV_err, of probabilities in fp16 that are rounded as 2^15 times themselves
        self.dV_fine = out(self.dV, add * group((half + rel) * Pt @ G.abs()) + (rows * 2.0 ** -24) * group(Pt @ G.abs()) +
                           tiny * 2.0 ** -15 * group(G.abs().sum(2, keepdim=True).expand(B, Hq, N, d)))
        sizeS = dS.abs()
        self.dQ_err = out(self.dQ, scale * (add * (dSerr @ Kg.abs()) + N * 2.0 ** -24 * (sizeS @ Kg.abs()) +
                                            tiny * Kg.abs().sum(2, keepdim=True)))
        self.dK_err = out(self.dK, scale * group(
            add * (dSerr.transpose(2, 3) @ Q.abs()) + rows * 2.0 ** -24 * (sizeS.transpose(2, 3) @ Q.abs()) +
            tiny * Q.abs().sum(2, keepdim=True).expand(B, Hq, N, d)))
        # keys that do not count have gradients of exactly 0
        for t in (self.dK_err, self.dV_err):
            t.masked_fill_(~on[:, None], 0.0)
