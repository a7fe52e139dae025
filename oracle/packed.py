"""Float64 definitions of the operators on packed token rows (test infrastructure only):
head norms with rotary positions, and causal attention with grouped heads over packed
sequences.  Written sequence by sequence from the formulas; backward passes by reverse-mode
differentiation of them, tangents by forward-mode differentiation of both."""
from __future__ import annotations

import math

import torch

F64 = torch.float64


def positions(lens):
    return torch.cat([torch.arange(n) for n in lens] + [torch.zeros(0, dtype=torch.long)])


def rates(dims, base=10000.0, scaling="none", factor=1.0, orig_len=0, low=1.0, high=4.0):
    """Radians a position of each rotated pair."""
    if scaling == "base":
        base = base * factor ** (dims / (dims - 2))
    out = []
    for j in range(dims // 2):
        w = base ** (-2.0 * j / dims)
        if scaling == "linear":
            w /= factor
        if scaling == "bands":
            turns = orig_len * w / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - low) / (high - low)))
            w = keep * w + (1 - keep) * w / factor
        out.append(w)
    return torch.tensor(out, dtype=F64)


def rotate(x, pos, w, layout, mscale=1.0):
    """x [rows][heads][D]: the first 2 len(w) elements of each head turned by pos w."""
    R = 2 * len(w)
    ang = pos.to(F64)[:, None, None] * w
    c, s = torch.cos(ang) * mscale, torch.sin(ang) * mscale
    if layout == "half":
        a, b = x[..., :R // 2], x[..., R // 2:R]
        z = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        z = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([z, x[..., R:]], -1)


def qk_rope(x, gq, gk, Hq, Hkv, D, pos, w, layout, mscale=1.0, eps=1e-6):
    """Rows [q heads | k heads | other columns] in float64; gq = gk = None: no norm."""
    q, k, rest = x[:, :Hq * D], x[:, Hq * D:(Hq + Hkv) * D], x[:, (Hq + Hkv) * D:]
    out = []
    for t, g in ((q, gq), (k, gk)):
        t = t.unflatten(1, (-1, D))
        if g is not None:
            t = g * t * torch.rsqrt((t * t).mean(-1, keepdim=True) + eps)
        out.append(rotate(t, pos, w, layout, mscale).flatten(1))
    return torch.cat(out + [rest], 1)


def attention(q, k, v, Hq, Hkv, D, lens, scale):
    """(o [N][Hq D], lse [Hq][N]) of rows packed as lens."""
    G = Hq // Hkv
    os, ls, a = [], [], 0
    for n in lens:
        r = slice(a, a + n)
        a += n
        Q = q[r].unflatten(1, (Hq, D)).transpose(0, 1)
        K = k[r].unflatten(1, (Hkv, D)).transpose(0, 1).repeat_interleave(G, 0)
        V = v[r].unflatten(1, (Hkv, D)).transpose(0, 1).repeat_interleave(G, 0)
        S = scale * Q @ K.transpose(1, 2)
        S = S.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
        lse = torch.logsumexp(S, -1)
        os.append((torch.exp(S - lse[..., None]) @ V).transpose(0, 1).flatten(1))
        ls.append(lse)
    return torch.cat(os), torch.cat(ls, 1)


def window_pairs(lens, window, sinks, device="cpu"):
    """Which rows attend to which, [N][N]: a row of a sequence to itself, the window - 1 rows before
    it and the first sinks rows of the sequence up to itself."""
    n = torch.tensor(lens, dtype=torch.long, device=device)
    seq = torch.repeat_interleave(torch.arange(len(lens), device=device), n)
    place = torch.arange(len(seq), device=device) - (torch.cumsum(n, 0) - n)[seq]
    i, j = place[:, None], place[None, :]
    return (seq[:, None] == seq[None, :]) & (j <= i) & ((i - j < window) | (j < sinks))


def masked_attention(q, k, v, Hq, Hkv, D, pairs, scale):
    """(o [N][Hq D], lse [Hq][N]) of rows that attend where pairs [N][N] says so."""
    heads = lambda t, H: t.unflatten(1, (H, D)).transpose(0, 1)
    K, V = (heads(t, Hkv).repeat_interleave(Hq // Hkv, 0) for t in (k, v))
    S = (scale * heads(q, Hq) @ K.mT).masked_fill(~pairs, -math.inf)
    lse = torch.logsumexp(S, -1)
    return (torch.exp(S - lse[..., None]) @ V).transpose(0, 1).flatten(1), lse


def grads(f, prim, cot):
    """Gradients of <f(prim), cot>."""
    return torch.func.vjp(f, *prim)[1](cot)


def grads_dual(f, prim, cot, dprim, dcot):
    """(gradients, their tangents along dprim, dcot)."""
    return torch.func.jvp(lambda c, *p: grads(f, p, c), (cot, *prim), (dcot, *dprim))
