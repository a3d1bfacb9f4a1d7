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
