"""Plain implementation, in 64 bits, of attention with a learned relative position bias (Algorithms 1 and 2 on the biased
scores), one query head at a time."""
import math

import torch


def bucket_starts(num_buckets, max_distance, bidirectional):
    """(e, h, distances at which the buckets e + 1 .. h - 1 begin), from whole numbers: the first n with
    (n / e)^(h - e) >= (max_distance / e)^j."""
    h = num_buckets // 2 if bidirectional else num_buckets
    e = h // 2
    w = h - e
    starts, n = [], e
    for j in range(1, w):
        lo = max(e, int(e * (max_distance / e) ** (j / w)) - 2)
        n = max(n, lo)
        while n ** w * e ** j < max_distance ** j * e ** w:
            n += 1
        starts.append(n)
    return e, h, starts


def buckets(delta, num_buckets, max_distance, bidirectional):
    e, h, starts = bucket_starts(num_buckets, max_distance, bidirectional)
    n = delta.abs() if bidirectional else (-delta).clamp(min=0)
    s = torch.tensor(starts, dtype=torch.int64, device=delta.device)
    far = e + (n[..., None] >= s).sum(-1) if starts else torch.full_like(n, e)
    b = torch.where(n < e, n, far)
    return b + h * (delta > 0) if bidirectional else b


def scores(q, k, table, scale, nb, md, bidir, causal, offset=None):
    """x [Nq, Nk] of one head (q [Nq,d], k [Nk,d], table [nb]); -inf where not legal, and the buckets."""
    Nq, Nk = q.shape[0], k.shape[0]
    off = Nk - Nq if offset is None else offset
    delta = torch.arange(Nk, device=q.device)[None] - torch.arange(Nq, device=q.device)[:, None] - off
    bk = buckets(delta, nb, md, bidir)
    x = q @ k.T * scale + table[bk]
    if causal:
        x = torch.where(delta > 0, torch.full_like(x, -math.inf), x)
    return x, bk


def softmax_rows(x):
    """(p, lse); a row of nothing but -inf gets p = 0, lse = -inf."""
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[..., None])
    return p, lse


def head(q, k, v, table, do, scale, nb, md, bidir, causal, keep=None, lse=None, D=None):
    """Forward and backward of one head.  keep [Nq, Nk]: the retained pairs (None: all).  lse, D: given ones instead of the
    head's own (Algorithm 2 works on the forward's).  Returns a dict; the d* entries come with `do`."""
    x, bk = scores(q, k, table, scale, nb, md, bidir, causal)
    if keep is not None:
        x = torch.where(keep, x, torch.full_like(x, -math.inf))
    p, z = softmax_rows(x)
    if lse is not None:
        p = torch.exp(x - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
    out = dict(o=p @ v, lse=z, a=p @ v.abs(), x=x, bk=bk)
    if do is None:
        return out
    dp = do @ v.T
    D = (out["o"] * do).sum(-1) if D is None else D
    ds = p * (dp - D[:, None])
    sums = lambda t: torch.stack([(t * (bk == b)).sum() for b in range(nb)])  # noqa: E731
    out.update(dv=p.T @ do, dq=ds @ k * scale, dk=ds.T @ q * scale, dtable=sums(ds))
    # what the kernel's roundings can add to a bucket: P to bf16 (u p |dp - D|), and D from the bf16 output, which itself
    # comes from bf16 P (u (|o| + a) per channel)
    u = 2.0 ** -8
    dD = u * ((out["o"].abs() + out["a"]) * do.abs()).sum(-1)
    out["dtable_err"] = u * sums(p * (dp - D[:, None]).abs()) + sums(p * dD[:, None])
    return out


def alg1_mask(x, tau, L, Bq=128, Bk=128, shift=0):
    """Tiles that Algorithm 1 retains on scores x [Nq, Nk] (-inf: not legal): (mask [Tq, Tk] of 0 not legal / 1 skipped / 2
    retained, criterion [Tq, Tk]).  Query block i holds the rows q with Bq i <= q + shift < Bq (i + 1); L [Nq]."""
    Nq, Nk = x.shape
    Tq, Tk = -(-(Nq + shift) // Bq), -(-Nk // Bk)
    mask = torch.zeros((Tq, Tk), dtype=torch.int64)
    crit = torch.full((Tq, Tk), -math.inf, dtype=torch.float64)
    for i in range(Tq):
        r = slice(max(0, i * Bq - shift), min(Nq, (i + 1) * Bq - shift))
        m = torch.full((r.stop - r.start,), -math.inf, dtype=torch.float64, device=x.device)
        l = torch.zeros_like(m)
        for j in range(Tk - 1, -1, -1):
            t = x[r, j * Bk:(j + 1) * Bk]
            if bool((t == -math.inf).all()):
                continue
            top = t.max(1).values
            c = torch.where(l > 0, top - (m + l.log()) - torch.log(tau / L[r]), torch.full_like(top, math.inf))
            c = torch.where(top == -math.inf, torch.full_like(c, -math.inf), c)
            crit[i, j] = c.max().item()
            if crit[i, j] < 0:
                mask[i, j] = 1
                continue
            mask[i, j] = 2
            new = torch.maximum(m, top)
            l = l * torch.exp(m - new) + torch.exp(t - new[:, None]).sum(1)
            m = new
    return mask, crit


def expand(mask, Nq, Nk, shift=0, B=128):
    """Retained pairs [Nq, Nk] of a mask of tiles."""
    q = (torch.arange(Nq) + shift) // B
    k = torch.arange(Nk) // B
    return (mask == 2)[q][:, k]
