"""Operators around the attention path that take it to models with a relative position bias and to a served, paged cache.

A case is a dict of plain values; its ``kind`` names the operator:

  train    attention with a learned bias per bucket of relative positions: forward, and backward with the table's gradient
  packed   the same on packed sequences of different lengths
  encode   its forward alone
  decode   its form for one or several new tokens per sequence over a paged cache
  tables   block tables, slots and offsets of one serving step from the requests' lengths, behind the release of the
           pages of finished requests
  write    new keys and values into the pages of a bf16 cache
  write8   the same into an e4m3 cache with a scale per tile (or page), tiles that already hold keys among them

With ``own`` false ``run`` computes them from elementary torch operations.
"""
import math
import random

import torch

own = False


def listed():
    return [
        # one layer of a small decoder at a short context: latency of forward + backward
        dict(name="train_1k_d64", kind="train", B=1, Hq=2, Hkv=2, Nq=1024, Nk=1024, d=64, causal=True, bidir=False,
             buckets=32, maxdist=128),
        # ordinary training context, grouped heads, a bias that reaches far
        dict(name="train_8k_d128", kind="train", B=1, Hq=16, Hkv=4, Nq=8192, Nk=8192, d=128, causal=True, bidir=False,
             buckets=64, maxdist=2048),
        # an encoder's training batch of documents of different lengths in one row
        dict(name="train_packed", kind="packed", Hq=16, Hkv=16, seqs=9, longest=2000, lens=11, d=64, causal=False,
             bidir=True, buckets=32, maxdist=128),
        # encoder states of a batch of passages
        dict(name="encode_512", kind="encode", B=32, Hq=16, Hkv=16, Nq=512, Nk=512, d=64, causal=False, bidir=True,
             buckets=32, maxdist=128),
        # one step of a single conversation: latency
        dict(name="decode_single", kind="decode", B=1, Hq=32, Hkv=8, longest=2000, lens=1, page=16, Sq=1, d=128,
             bidir=False, buckets=32, maxdist=128),
        # a serving batch of conversations of different lengths, two tokens verified per step
        dict(name="decode_batch", kind="decode", B=32, Hq=32, Hkv=8, longest=16000, lens=7, page=128, Sq=2, d=128,
             bidir=False, buckets=32, maxdist=128),
        # one decode step of a serving batch: a token each, some requests finished
        dict(name="tables_step", kind="tables", B=64, page=16, longest=4000, most_new=1, lens=5),
        # admission of many prompts at once
        dict(name="tables_prompts", kind="tables", B=1000, page=64, longest=500, most_new=2000, lens=6),
        # the keys and values of one decode step
        dict(name="write_step", kind="write", B=64, most_new=1, longest=4000, page=16, Hkv=8, d=128, lens=2),
        # prefill chunks of several sequences behind cached prefixes
        dict(name="write_prefill", kind="write", B=9, most_new=6000, longest=9000, page=64, Hkv=8, d=128, lens=3),
        # the decode step over an e4m3 cache: most tiles hold keys already
        dict(name="write8_step", kind="write8", B=64, most_new=1, longest=4000, page=128, Hkv=8, d=128, lens=2),
        # the prefill chunks over an e4m3 cache
        dict(name="write8_prefill", kind="write8", B=9, most_new=6000, longest=9000, page=64, Hkv=8, d=128, lens=3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["train", "packed", "encode", "decode", "decode", "tables", "write", "write8"])
    c = dict(kind=kind)
    if kind in ("train", "packed", "encode"):
        heads = rng.choice([(2, 2), (8, 2), (16, 4), (16, 16)])
        causal = rng.random() < 0.5
        buckets = rng.choice([8, 16, 32, 32, 64])
        c.update(Hq=heads[0], Hkv=heads[1], d=rng.choice([64, 64, 96, 128]), causal=causal,
                 bidir=(not causal) or rng.random() < 0.2, buckets=buckets, maxdist=_log(rng, 2 * buckets, 4096))
        if kind == "packed":
            c.update(seqs=rng.randint(2, 12), longest=_log(rng, 100, 2000), lens=rng.randrange(1000))
        else:
            n = _log(rng, 100, 5000)
            c.update(B=max(1, min(rng.choice([1, 2, 8, 32]), (5000 // n) ** 2)), Nk=n,
                     Nq=n if rng.random() < 0.7 else rng.randint(1, n))
    elif kind == "decode":
        heads = rng.choice([(8, 8), (8, 2), (32, 8)])
        c.update(B=_log(rng, 1, 32), Hq=heads[0], Hkv=heads[1], longest=_log(rng, 200, 16000), lens=rng.randrange(1000),
                 page=rng.choice([16, 64, 128, 256]), Sq=rng.choice([1, 1, 2, 4]), d=rng.choice([64, 128, 128]),
                 bidir=rng.random() < 0.3, buckets=rng.choice([16, 32, 64]), maxdist=_log(rng, 128, 4096))
    elif kind == "tables":
        c.update(B=_log(rng, 1, 1000), page=rng.choice([8, 16, 64, 128, 256]), longest=_log(rng, 10, 4000),
                 most_new=rng.choice([1, 1, 4, _log(rng, 10, 2000)]), lens=rng.randrange(1000))
    else:
        small = rng.random() < 0.5
        c.update(B=_log(rng, 1, 64) if small else _log(rng, 1, 9), most_new=rng.choice([1, 1, 4]) if small else _log(rng, 50, 6000),
                 longest=_log(rng, 200, 9000), page=rng.choice([16, 64, 128, 256]), Hkv=rng.choice([1, 2, 8]),
                 d=rng.choice([64, 128, 128]), lens=rng.randrange(1000))
    return c


# ------------------------------------------------------------------------------------------------ sizes of a case

def _lengths(n, longest, which):
    """n lengths of up to `longest`, the first one that long, one of them 1."""
    r = random.Random(which)
    out = [max(1, int(longest * r.uniform(0.05, 1.0))) for _ in range(n)]
    out[0] = longest
    if n > 2:
        out[n // 2] = 1
    return out


def _serving(case):
    """(keys that each request holds, its new tokens, whether it has finished) of a `tables`, `write` or `write8` case."""
    r = random.Random(case["lens"] * 7 + 1)
    held = [r.randint(0, case["longest"]) for _ in range(case["B"])]
    if case["most_new"] > 8:
        new = [r.randint(0, case["most_new"]) for _ in range(case["B"])]
        new[0] = case["most_new"]
    else:
        new = [case["most_new"]] * case["B"]
    done = [r.random() < 0.1 for _ in range(case["B"])]
    return held, new, done


def _pairs(case):
    """(visible query-key pairs of one head, query rows, key rows) of an attention case."""
    if case["kind"] == "packed":
        lens = _lengths(case["seqs"], case["longest"], case["lens"])
        return sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lens), sum(lens), sum(lens)
    q, k = case["Nq"], case["Nk"]
    return case["B"] * (q * (k - q) + q * (q + 1) // 2 if case["causal"] else q * k), case["B"] * q, case["B"] * k


def work(case):
    kind = case["kind"]
    if kind in ("train", "packed", "encode"):
        pairs, nq, nk = _pairs(case)
        Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
        flops, nbytes = 4 * pairs * d * Hq, 2 * d * (2 * nq * Hq + 2 * nk * Hkv) + 4 * nq * Hq + 2 * case["buckets"] * Hq
        if kind != "encode":   # five products more; reads dO, writes dQ, dK, dV and the table's gradient
            flops += 10 * pairs * d * Hq
            nbytes += 2 * d * (2 * nq * Hq + 2 * nk * Hkv) + 2 * case["buckets"] * Hq
        return {"bytes": nbytes, "flops": flops}
    if kind == "decode":
        keys = sum(max(n, case["Sq"]) for n in _lengths(case["B"], case["longest"], case["lens"]))
        rows = case["B"] * case["Sq"] * case["Hq"]
        return {"bytes": 4 * keys * case["Hkv"] * case["d"] + rows * (4 * case["d"] + 4) + 2 * case["buckets"] * case["Hq"],
                "flops": 4 * keys * case["Sq"] * case["Hq"] * case["d"]}
    held, new, done = _serving(case)
    total, ps = sum(new), case["page"]
    if kind == "tables":
        held2 = [0 if f else n for n, f in zip(held, done)]
        fresh = sum(-(-(h + n) // ps) - -(-h // ps) for h, n in zip(held2, new))
        back = sum(-(-h // ps) for h, f in zip(held, done) if f)
        return {"bytes": 4 * (3 * len(held) + 2 * fresh + 2 * back + 2 * len(held)) + 8 * total, "flops": 0}
    elements = 2 * total * case["Hkv"] * case["d"]
    return {"bytes": elements * (4 if kind == "write" else 3) + 8 * total, "flops": 0 if kind == "write" else 2 * elements}


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    kind = case["kind"]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=dev).to(torch.bfloat16)

    if kind in ("train", "packed", "encode"):
        s = dict(case=case, scale=1.0 / math.sqrt(case["d"]))
        if kind == "packed":
            lens = _lengths(case["seqs"], case["longest"], case["lens"])
            s["cu"] = torch.tensor([0] + lens, device=dev).cumsum(0).to(torch.int32)
            s["longest"] = max(lens)
            B, nq, nk = 1, sum(lens), sum(lens)
        else:
            B, nq, nk = case["B"], case["Nq"], case["Nk"]
        s["q"], s["k"], s["v"] = randn(B, nq, case["Hq"], case["d"]), randn(B, nk, case["Hkv"], case["d"]), randn(B, nk, case["Hkv"], case["d"])
        s["do"] = randn(B, nq, case["Hq"], case["d"])
        s["table"] = randn(case["buckets"], case["Hq"])
        return s
    if kind == "decode":
        lens = [max(n, case["Sq"]) for n in _lengths(case["B"], case["longest"], case["lens"])]
        ps = case["page"]
        per = [-(-n // ps) for n in lens]
        pool = sum(per) + 3
        order = torch.randperm(pool, generator=gen, device=dev).to(torch.int32)
        table = torch.full((case["B"], max(per)), -1, device=dev, dtype=torch.int32)
        at = 0
        for b, n in enumerate(per):      # the pages of a request lie anywhere in the pool
            table[b, :n] = order[at:at + n]
            at += n
        return dict(case=case, scale=1.0 / math.sqrt(case["d"]), q=randn(case["B"], case["Sq"], case["Hq"], case["d"]),
                    kpages=randn(pool, ps, case["Hkv"], case["d"]), vpages=randn(pool, ps, case["Hkv"], case["d"]),
                    block_table=table, seqlens=torch.tensor(lens, device=dev, dtype=torch.int32), longest=max(lens),
                    table=randn(case["buckets"], case["Hq"]))
    held, new, done = _serving(case)
    ps, B, total = case["page"], case["B"], sum(new)
    per = [-(-n // ps) for n in held]
    grown = [-(-(h + n) // ps) for h, n in zip(held, new)]
    pool = sum(grown) + 5
    order = torch.randperm(pool, generator=gen, device=dev).to(torch.int32)
    if kind == "tables":
        width = max(max(grown), 1)
        table = torch.zeros((B, width), device=dev, dtype=torch.int32)
        start = torch.tensor([0] + per, device=dev).cumsum(0)[:-1]
        x = torch.arange(width, device=dev)
        mine = x[None] < torch.tensor(per, device=dev)[:, None]
        table[mine] = order[(start[:, None] + x[None])[mine]]
        free = torch.zeros(pool, device=dev, dtype=torch.int32)
        left = pool - sum(per)
        free[:left] = order[sum(per):]
        return dict(case=case, block_table=table, free_pages=free, total=total,
                    free_count=torch.tensor([left], device=dev, dtype=torch.int32),
                    seqlens=torch.tensor(held, device=dev, dtype=torch.int32),
                    new=torch.tensor(new, device=dev, dtype=torch.int32), done=torch.tensor(done, device=dev))
    # slots of the new rows, request by request, behind the keys that it holds; the last request is refused (slot -1)
    h, n = torch.tensor(held, device=dev), torch.tensor(new, device=dev)
    first = torch.tensor([0] + grown, device=dev).cumsum(0)[:-1]
    seq = torch.repeat_interleave(torch.arange(B, device=dev), n, output_size=total)
    pos = h[seq] + torch.arange(total, device=dev) - (n.cumsum(0) - n)[seq]
    slots = order[first[seq] + pos // ps].to(torch.int64) * ps + pos % ps
    if B > 1:
        slots = torch.where(seq == B - 1, torch.full_like(slots, -1), slots)
    rows = (total, case["Hkv"], case["d"])
    s = dict(case=case, slots=slots, k=randn(*rows), v=randn(*rows))
    page = (pool, ps, case["Hkv"], case["d"])
    if kind == "write":
        s["kpages"], s["vpages"] = randn(*page), randn(*page)
    else:
        # a tenth of the rows are larger than what their tile holds
        big = torch.rand((total, 1, 1), generator=gen, device=dev) < 0.1
        for x in ("k", "v"):
            s[x] = torch.where(big, s[x] * 4, s[x])
            s[x + "pages"] = (torch.randn(page, generator=gen, device=dev) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
            s[x + "scale"] = torch.rand((pool, case["Hkv"], max(1, ps // 128)), generator=gen, device=dev) * 0.01 + 0.005
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(state)
    if kind in ("train", "packed", "encode"):
        return _attention(state)
    return {"decode": _decode, "tables": _tables, "write": _write, "write8": _write8}[kind](state)


def _own(s):
    from paper_2609_32712_b200 import mala
    c, kind = s["case"], s["case"]["kind"]
    if kind in ("train", "encode", "packed", "decode"):
        bias = mala.RelativeBias(s["table"], max_distance=c["maxdist"], bidirectional=c["bidir"])
    if kind in ("train", "encode"):
        o, lse, _ = mala.fwd_bias(s["q"], s["k"], s["v"], bias, s["scale"], 0.0, causal=c["causal"])
        if kind == "encode":
            return o, lse
        return (o, lse) + mala.bwd_bias(s["q"], s["k"], s["v"], o, s["do"], lse, bias, s["scale"], 0.0, causal=c["causal"])[:4]
    if kind == "packed":
        n = s["longest"]
        o, lse, _ = mala.fwd_varlen_bias(s["q"], s["k"], s["v"], s["cu"], s["cu"], n, n, bias, s["scale"], 0.0, causal=c["causal"])
        return (o, lse) + mala.bwd_varlen_bias(s["q"], s["k"], s["v"], o, s["do"], lse, s["cu"], s["cu"], n, n, bias, s["scale"], 0.0,
                                               causal=c["causal"])[:4]
    if kind == "decode":
        splits = mala.decode_suggest_splits(c["B"], c["Hkv"], s["longest"])
        return mala.decode_paged_bias(s["q"], s["kpages"], s["vpages"], s["block_table"], s["seqlens"], bias, s["scale"], 0.0, splits)[:2]
    if kind == "tables":
        table, free = s["block_table"].clone(), s["free_pages"].clone()    # (a step changes them: the next pass starts from these again)
        held, count = mala.release_pages(s["done"], s["seqlens"], table, free, s["free_count"], c["page"])
        cu, lens, slots, left = mala.page_tables(held, s["new"], table, free, count, c["page"], s["total"])
        return table, free, cu, lens, slots, left
    if kind == "write":
        mala.cache_write(s["k"], s["v"], s["slots"], s["kpages"], s["vpages"])
        return s["kpages"], s["vpages"]
    mala.cache_write_fp8(s["k"], s["v"], s["slots"], s["kpages"], s["vpages"], s["kscale"], s["vscale"])
    return s["kpages"], s["kscale"], s["vpages"], s["vscale"]


def _bucket(delta, buckets, maxdist, bidir):
    """Bucket of a relative position (key - query): half of a side's buckets hold one distance each, the rest grow with
    its logarithm.  The logarithms in 64 bits, and a distance at a border belongs to the bucket that begins there."""
    side = buckets // 2 if bidir else buckets
    n = delta.abs() if bidir else (-delta).clamp(min=0)
    exact = side // 2
    far = exact + ((n.clamp(min=1).double() / exact).log() / math.log(maxdist / exact) * (side - exact) + 1e-9).floor().long()
    b = torch.where(n < exact, n, far.clamp(max=side - 1))
    return torch.where(delta > 0, b + side, b) if bidir else b


def _attention(s):
    c = s["case"]
    q, k, v, do = s["q"].float(), s["k"].float(), s["v"].float(), s["do"].float()
    dev = q.device
    if c["kind"] == "packed":   # one padded row per sequence
        cu = s["cu"].long()
        n, M = cu[1:] - cu[:-1], s["longest"]
        x = torch.arange(M, device=dev)
        real = x[None] < n[:, None]
        at = (cu[:-1, None] + x[None]).clamp(max=q.shape[1] - 1)
        q, k, v, do = (t[0][at] * real[:, :, None, None] for t in (q, k, v, do))
        keep = real[:, None, :] & real[:, :, None]
    B, Nq, Hq, d = q.shape
    Nk, Hkv = k.shape[1], k.shape[2]
    G = Hq // Hkv
    q, do = (t.view(B, Nq, Hkv, G, d).permute(0, 2, 3, 1, 4) for t in (q, do))   # [B, Hkv, G, Nq, d]
    k, v = (t.permute(0, 2, 1, 3)[:, :, None] for t in (k, v))                   # [B, Hkv, 1, Nk, d]
    delta = torch.arange(Nk, device=dev)[None] - torch.arange(Nq, device=dev)[:, None] - (Nk - Nq)
    bias = s["table"].float().t()[:, _bucket(delta, c["buckets"], c["maxdist"], c["bidir"])].view(Hkv, G, Nq, Nk)
    x = (q @ k.transpose(-1, -2)) * s["scale"] + bias
    del bias
    if c["causal"]:
        x.masked_fill_(delta > 0, -math.inf)
    if c["kind"] == "packed":
        x.masked_fill_(~keep[:, None, None, :, :] & real[:, None, None, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    x = (x - m).exp_()
    l = x.sum(-1, keepdim=True)
    p = x.div_(l)
    o = p @ v
    lse = (m + l.log())[..., 0].reshape(B, Hq, Nq)

    def rows(t, heads, length):   # [B, heads, length, d] as the call's layout
        t = t.reshape(B, heads, length, d).permute(0, 2, 1, 3)
        if c["kind"] == "packed":
            row = torch.arange(s["q"].shape[1], device=dev)
            seq = torch.searchsorted(cu[1:], row, right=True)
            t = t[seq, row - cu[seq]][None]
        return t.to(torch.bfloat16)
    out = rows(o, Hq, Nq)
    if c["kind"] == "packed":
        row = torch.arange(s["q"].shape[1], device=dev)
        seq = torch.searchsorted(cu[1:], row, right=True)
        lse = lse.permute(1, 0, 2)[:, seq, row - cu[seq]]
    if c["kind"] == "encode":
        return out, lse
    dv = (p.transpose(-1, -2) @ do).sum(2)
    ds = do @ v.transpose(-1, -2)
    ds.sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    del p, x
    dq = (ds @ k) * s["scale"]
    dk = (ds.transpose(-1, -2) @ q).sum(2) * s["scale"]
    # sums along the diagonals: the rows back to front, each moved one column further than the one before
    skew = torch.nn.functional.pad(ds.sum(0).reshape(Hq, Nq, Nk).flip(1), (0, Nq)).reshape(Hq, -1)
    del ds
    L = Nq + Nk - 1
    diag = skew[:, :Nq * L].view(Hq, Nq, L).sum(1, dtype=torch.float64)
    which = _bucket(torch.arange(L, device=dev) - (Nk - 1), c["buckets"], c["maxdist"], c["bidir"])
    dtable = ((which[:, None] == torch.arange(c["buckets"], device=dev)).double().t() @ diag.t()).to(torch.bfloat16)
    return out, lse, rows(dq, Hq, Nq), rows(dk, Hkv, Nk), rows(dv, Hkv, Nk), dtable


def _decode(s):
    c = s["case"]
    q, n = s["q"].float(), s["seqlens"].long()
    B, Sq, Hq, d = q.shape
    Hkv, ps = c["Hkv"], c["page"]
    pages = s["block_table"].long().clamp(min=0)
    k, v = (t[pages].float().view(B, -1, Hkv, d).permute(0, 2, 1, 3) for t in (s["kpages"], s["vpages"]))   # [B, Hkv, keys, d]
    key = torch.arange(k.shape[2], device=q.device)
    at = n[:, None] - Sq + torch.arange(Sq, device=q.device)[None]                                           # position of each token
    delta = key[None, None] - at[:, :, None]
    bias = s["table"].float()[_bucket(delta, c["buckets"], c["maxdist"], c["bidir"])]                        # [B, Sq, keys, Hq]
    bias = bias.permute(0, 3, 1, 2).view(B, Hkv, Hq // Hkv, Sq, -1)
    qh = q.view(B, Sq, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    x = (qh @ k.transpose(-1, -2)).view(bias.shape) * s["scale"] + bias
    x = x.masked_fill((delta > 0)[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = (x - m).exp()
    l = p.sum(-1, keepdim=True)
    o = ((p / l).view(B, Hkv, -1, p.shape[-1]) @ v).view(B, Hkv, Hq // Hkv, Sq, d)
    lse = (m + l.log())[..., 0].permute(0, 3, 1, 2).reshape(B, Sq, Hq)
    return o.permute(0, 3, 1, 2, 4).reshape(B, Sq, Hq, d).to(torch.bfloat16), lse[:, 0] if Sq == 1 else lse


def _tables(s):
    ps, table, free = s["case"]["page"], s["block_table"].long(), s["free_pages"].long()
    B, width = table.shape
    x = torch.arange(width, device=table.device)[None]
    # finished requests give their pages back, in their order, behind the free ones
    n, done, count = s["seqlens"].long(), s["done"], s["free_count"].long()
    back = torch.where(done, (n + ps - 1) // ps, torch.zeros_like(n))
    at = count + (back.cumsum(0) - back)[:, None] + x
    free = torch.cat([free, free[:1]]).scatter(0, torch.where(x < back[:, None], at, torch.full_like(at, free.numel())).flatten(), table.flatten())[:-1]
    free_pages = free.to(torch.int32)
    count = count + back.sum()
    n = torch.where(done, torch.zeros_like(n), n)
    # pages for the new tokens, off the end of the list
    new = s["new"].long()
    have, fits = (n + ps - 1) // ps, n + new <= width * ps
    need = torch.where(fits, (n + new + ps - 1) // ps - have, torch.zeros_like(n))
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= count))
    nth = (upto - need)[:, None] + x - have[:, None]
    fresh = ok[:, None] & (x >= have[:, None]) & (x < (have + need)[:, None])
    table = torch.where(fresh, free[(count - 1 - nth).clamp(0, free.numel() - 1)], table)
    left = count - (need * ok).sum()
    cu = torch.nn.functional.pad(new.cumsum(0), (1, 0))
    row = torch.arange(s["total"], device=table.device)
    seq = torch.searchsorted(cu[1:], row, right=True).clamp(max=B - 1)
    pos = n[seq] + row - cu[seq]
    slots = torch.where(ok[seq] & (row < cu[-1]), table[seq, (pos // ps).clamp(max=width - 1)] * ps + pos % ps, torch.full_like(row, -1))
    return table.to(torch.int32), free_pages, cu.to(torch.int32), torch.where(ok, n + new, n).to(torch.int32), slots, left.to(torch.int32)


def _write(s):
    ok = s["slots"] >= 0
    at = s["slots"][ok]
    s["kpages"].view(-1, *s["k"].shape[1:])[at] = s["k"][ok]
    s["vpages"].view(-1, *s["v"].shape[1:])[at] = s["v"][ok]
    return s["kpages"], s["vpages"]


def _write8(s):
    ps = s["case"]["page"]
    unit = min(ps, 128)
    ok = s["slots"] >= 0
    at = s["slots"][ok]
    units, back = torch.unique(at // unit, return_inverse=True)      # the tiles (or pages) that get new keys
    new = torch.zeros((units.numel(), unit), device=at.device, dtype=torch.bool)
    new[back, at % unit] = True
    held = torch.arange(unit, device=at.device)[None] < new.long().argmax(1)[:, None]   # keys there before
    return (*_write8_one(s["k"][ok].float(), s["kpages"], s["kscale"], at, units, back, new, held),
            *_write8_one(s["v"][ok].float(), s["vpages"], s["vscale"], at, units, back, new, held))


def _write8_one(x, pages, scale, at, units, back, new, held):
    P, ps, H, d = pages.shape
    unit, per = new.shape[1], scale.shape[2]
    rows = torch.zeros((units.numel(), unit, H, d), device=x.device)
    rows[back, at % unit] = x
    top = rows.abs().amax((1, 3)) / 448.0                            # [units, H]
    before = scale[units // per, :, units % per]
    after = torch.where(new[:, :1], torch.where(top > 0, top, torch.ones_like(top)), torch.maximum(before, top))
    store = pages.view(torch.uint8).view(-1, unit, H, d)
    codes = store[units].view(torch.float8_e4m3fn).float()
    moved = held[:, :, None] & (after > before)[:, None]
    codes = torch.where(moved[..., None], (codes * before[:, None, :, None]) / after[:, None, :, None], codes)
    codes = torch.where(new[:, :, None, None], rows / after[:, None, :, None], codes)
    store[units] = codes.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    scale[units // per, :, units % per] = after
    return pages, scale


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("train", "packed", "encode"):
        return _exact_attention(s)
    if kind == "decode":
        return _exact_decode(s)
    if kind == "write8":
        return _exact_write8(s)
    if kind == "write":
        return tuple(_exact_copy(s[x], s[x + "pages"], s["slots"]) for x in ("k", "v"))
    return None      # whole numbers


def _exact_buckets(lo, hi, c, device):
    """Buckets of the relative positions lo .. hi, from the powers of the distances as whole numbers."""
    side = c["buckets"] // 2 if c["bidir"] else c["buckets"]
    e = side // 2
    w = side - e
    starts = []                    # the distance at which bucket e + j begins: the first n with (n/e)^w >= (maxdist/e)^j
    for j in range(1, w):
        n = max(e, int(e * (c["maxdist"] / e) ** (j / w)) - 2)
        while n ** w * e ** j < c["maxdist"] ** j * e ** w:
            n += 1
        starts.append(n)
    starts = torch.tensor(starts, device=device, dtype=torch.int64)
    delta = torch.arange(lo, hi + 1, device=device)
    n = delta.abs() if c["bidir"] else -delta.clamp(max=0)
    b = torch.where(n < e, n, e + torch.bucketize(n, starts, right=True))
    return b + side * (delta > 0) if c["bidir"] else b


def _exact_attention(s):
    c = s["case"]
    q, k, v, do = (s[x].double() for x in ("q", "k", "v", "do"))
    G, dev = c["Hq"] // c["Hkv"], q.device
    table = s["table"].double()
    o, dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dtable = torch.zeros_like(table)
    if c["kind"] == "packed":
        cu = s["cu"].tolist()
        parts = [(0, slice(a, b), slice(a, b)) for a, b in zip(cu, cu[1:])]
        lse = torch.zeros((c["Hq"], q.shape[1]), device=dev, dtype=torch.float64)
    else:
        parts = [(b, slice(0, c["Nq"]), slice(0, c["Nk"])) for b in range(c["B"])]
        lse = torch.zeros((c["B"], c["Hq"], c["Nq"]), device=dev, dtype=torch.float64)
    for b, rq, rk in parts:
        nq, nk = rq.stop - rq.start, rk.stop - rk.start
        near = _exact_buckets(1 - nk, nk - 1, c, dev) if nk >= nq else _exact_buckets(1 - nq, nq - 1, c, dev)
        far = max(nk, nq) - 1
        delta = torch.arange(nk, device=dev)[None] - torch.arange(nk - nq, nk, device=dev)[:, None]
        bucket = near[delta + far]
        for h in range(c["Hq"]):
            qh, kh, vh, gh = q[b, rq, h], k[b, rk, h // G], v[b, rk, h // G], do[b, rq, h]
            x = qh @ kh.T * s["scale"] + table[:, h][bucket]
            if c["causal"]:
                x = x.where(delta <= 0, -math.inf)
            z = torch.logsumexp(x, 1)
            p = torch.exp(x - z[:, None])
            o[b, rq, h] = p @ vh
            if c["kind"] == "packed":
                lse[h, rq] = z
            else:
                lse[b, h] = z
            if c["kind"] == "encode":
                continue
            dv[b, rk, h // G] += p.T @ gh
            t = p * (gh @ vh.T)
            ds = t - p * t.sum(1, keepdim=True)
            dq[b, rq, h] = ds @ kh * s["scale"]
            dk[b, rk, h // G] += ds.T @ qh * s["scale"]
            for j in range(c["buckets"]):
                dtable[j, h] += (ds * (bucket == j)).sum()
    return (o, lse) if c["kind"] == "encode" else (o, lse, dq, dk, dv, dtable)


def _exact_decode(s):
    c = s["case"]
    Sq, G, ps, dev = c["Sq"], c["Hq"] // c["Hkv"], c["page"], s["q"].device
    o = torch.zeros_like(s["q"], dtype=torch.float64)
    lse = torch.zeros(o.shape[:3], device=dev, dtype=torch.float64)
    for b, n in enumerate(s["seqlens"].tolist()):
        pages = s["block_table"][b, :-(-n // ps)].long()
        k, v = (s[x][pages].reshape(-1, c["Hkv"], c["d"])[:n].double().repeat_interleave(G, 1) for x in ("kpages", "vpages"))
        for t in range(Sq):
            seen = n - Sq + t + 1
            bias = s["table"].double()[_exact_buckets(1 - seen, 0, c, dev)]
            x = torch.einsum("hd,nhd->nh", s["q"][b, t].double(), k[:seen]) * s["scale"] + bias
            lse[b, t] = torch.logsumexp(x, 0)
            o[b, t] = torch.einsum("nh,nhd->hd", torch.softmax(x, 0), v[:seen])
    return o, lse[:, 0] if Sq == 1 else lse


def _exact_copy(rows, pages, slots):
    out = pages.double()
    for lo in range(0, slots.numel(), 1024):      # (a few rows at a time: the rows without a place are left out)
        part = slots[lo:lo + 1024]
        out.view(-1, *rows.shape[1:])[part[part >= 0]] = rows[lo:lo + 1024][part >= 0].double()
    return out


def _exact_write8(s):
    """Codes before their rounding to 8 bits, and scales."""
    P, ps, H, d = s["kpages"].shape
    unit = min(ps, 128)
    slots = s["slots"].cpu()
    rows = torch.nonzero(slots >= 0)[:, 0]
    u, back = torch.unique(slots[rows] // unit, return_inverse=True)
    out = []
    for x, pages, scale in ((s["k"], s["kpages"], s["kscale"]), (s["v"], s["vpages"], s["vscale"])):
        old = scale.double().permute(0, 2, 1).reshape(-1, H)
        codes = pages.double().reshape(-1, unit, H, d)
        dev = old.device
        ud, bd, rd = u.to(dev), back.to(dev), rows.to(dev)
        xs = x.double()[rd]
        a = torch.zeros((u.numel(), H), device=dev, dtype=torch.float64)
        a.scatter_reduce_(0, bd[:, None].expand(-1, H), xs.abs().amax(2) / 448, "amax")
        least = torch.full((u.numel(),), unit, device=dev).scatter_reduce(0, bd, s["slots"][rd] % unit, "amin")
        now = torch.where((least == 0)[:, None], torch.where(a > 0, a, 1.0), torch.maximum(a, old[ud]))
        ratio = torch.where(least[:, None] > 0, old[ud] / now, 1.0)
        held = (torch.arange(unit, device=dev)[None] < least[:, None])[:, :, None, None]
        codes[ud] = torch.where(held, codes[ud] * ratio[:, None, :, None], codes[ud])
        flat = codes.view(-1, H, d)
        flat[s["slots"][rd]] = xs / now[bd][:, :, None]
        new = old.clone()
        new[ud] = now
        out.append((codes.view(P, ps, H, d), new.view(P, -1, H).permute(0, 2, 1).contiguous()))
    return *out[0], *out[1]
