"""Rotary positions with a norm of each head in front, their gradients, and reads of a paged cache, in 64 bits and from the formulas (no
code of the library)."""
import math

import torch


def split(y, R, interleaved):
    return (y[..., 0:R:2], y[..., 1:R:2]) if interleaved else (y[..., :R // 2], y[..., R // 2:R])


def turn(y, pos, inv_freq, interleaved=False, magnitude=1.0, sense=1.0):
    """y [..., rows, H, d] (64 bits) at positions [..., rows]."""
    R = 2 * inv_freq.numel()
    a = (pos.double()[..., None] * inv_freq.double().to(y.device))[..., None, :]
    c, s = magnitude * a.cos(), sense * magnitude * a.sin()
    y1, y2 = split(y, R, interleaved)
    z1, z2 = y1 * c - y2 * s, y2 * c + y1 * s
    z = torch.stack([z1, z2], -1).flatten(-2) if interleaved else torch.cat([z1, z2], -1)
    return torch.cat([z, y[..., R:]], -1)


def normed(x, w, eps):
    x = x.double()
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return n if w is None else n * w.double()


def forward(x, pos, inv_freq, interleaved=False, magnitude=1.0, eps=None, w=None):
    y = x.double() if eps is None else normed(x, w, eps)
    return turn(y, pos, inv_freq, interleaved, magnitude)


def size(x, pos, inv_freq, interleaved=False, magnitude=1.0, eps=None, w=None):
    """What a rotation's fp32 errors are relative to: the sum of the magnitudes of an output's two terms."""
    y = (x.double() if eps is None else normed(x, w, eps)).abs()
    R = 2 * inv_freq.numel()
    y1, y2 = split(y, R, interleaved)
    z = magnitude * (y1 + y2)
    z = torch.stack([z, z], -1).flatten(-2) if interleaved else torch.cat([z, z], -1)
    return torch.cat([z, y[..., R:]], -1)


def backward(dy, x, pos, inv_freq, interleaved=False, magnitude=1.0, eps=None, w=None):
    """(dx, dw or None, g n as a check of dw's terms)."""
    g = turn(dy.double(), pos, inv_freq, interleaved, magnitude, -1.0)
    if eps is None:
        return g, None, None
    x = x.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n = x * r
    gw = g if w is None else g * w.double()
    dx = r * (gw - n * (gw * n).mean(-1, keepdim=True))
    return dx, (g * n).flatten(0, -2).sum(0), (g * n).abs().flatten(0, -2).sum(0)


def backward_size(dy, x, pos, inv_freq, interleaved=False, magnitude=1.0, eps=None, w=None):
    g = size(dy, pos, inv_freq, interleaved, magnitude)
    if eps is None:
        return g
    x = x.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n, gw = x * r, g if w is None else g * w.double().abs()
    return r * (gw + n.abs() * (gw * n.abs()).mean(-1, keepdim=True))


def packed_positions(cu_q, cu_k, total, queries):
    """Positions of packed rows (None where no sequence has the row)."""
    out = [None] * total
    for b in range(len(cu_q) - 1):
        nq, nk = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        at, n, first = (cu_q[b], nq, nk - nq) if queries else (cu_k[b], nk, 0)
        for x in range(n):
            out[at + x] = first + x
    return out


def values(pages, scale, table, n, ps):
    """Keys or values of one request in 64 bits, [n, Hkv, d]: pages bf16, or codes with scales [num_pages, Hkv, units]."""
    out = []
    for x in range(n):
        page, at = int(table[x // ps]), x % ps
        row = pages[page, at].double()
        out.append(row if scale is None else row * scale[page, :, at // 128].double()[:, None])
    return torch.stack(out) if out else pages.new_zeros((0, *pages.shape[2:]), dtype=torch.float64)


def attention(q, k, v, scale):
    """Causal attention of the last len(q) of len(k) positions, one head, 64 bits: (o, lse, sum of p |v|)."""
    x = q @ k.T * scale
    x = x.masked_fill(torch.ones_like(x, dtype=torch.bool).triu(len(k) - len(q) + 1), -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse[:, None])
    return p @ v, lse, p @ v.abs()
