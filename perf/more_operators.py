"""Rotary positions around the attention path, and an e4m3 cache that prompts can be read from.

A case is a dict of plain values; its ``kind`` names the operator:

  train    rotary positions of q and k, forward and backward, with a root-mean-square norm of each head in front or without
  packed   the same on packed sequences of different lengths
  rotate   the forward alone, at given positions
  step     rotary positions of a serving step's q and k, the keys and the values going into the pages of a bf16 cache
  step8    the same into an e4m3 cache with a scale per tile (or page), tiles that already hold keys among them
  read     keys and values of requests out of the pages of a bf16 cache, packed
  read8    the same out of an e4m3 cache
  prefill8 attention of prompts' chunks over an e4m3 cache (their own keys among it)

With ``own`` false ``run`` computes them from elementary torch operations.
"""
import math
import random

import torch

own = False

EPS = 1e-6


def listed():
    return [
        # one layer of a small decoder at a short context: latency of forward + backward
        dict(name="train_1k_d64", kind="train", B=1, N=1024, Hq=2, Hkv=2, d=64, rotary=64, pairs="halves", norm=False,
             base=10000.0, scaling="", start=0),
        # a long context, grouped heads, normed heads, frequencies scaled for it
        dict(name="train_32k_norm", kind="train", B=1, N=32768, Hq=32, Hkv=8, d=128, rotary=128, pairs="halves", norm=True,
             base=500000.0, scaling="yarn", start=0),
        # documents of different lengths in one row
        dict(name="packed_norm", kind="packed", seqs=9, longest=2000, lens=11, Hq=16, Hkv=4, d=128, rotary=128, pairs="halves",
             norm=True, base=10000.0, scaling=""),
        # hidden states of a batch far inside long documents, half of the head rotated, neighbours paired
        dict(name="rotate_far_partial", kind="rotate", B=8, N=4096, Hq=16, Hkv=4, d=128, rotary=64, pairs="neighbours", norm=False,
             base=10000.0, scaling="linear", start=700001),
        # one decode step of a serving batch: a token each
        dict(name="step_decode", kind="step", B=64, most_new=1, longest=4000, page=16, Hq=32, Hkv=8, d=128, rotary=128,
             pairs="halves", norm=False, base=500000.0, scaling="", lens=2),
        # prefill chunks of several sequences behind cached prefixes, normed heads
        dict(name="step_prefill", kind="step", B=9, most_new=6000, longest=9000, page=64, Hq=32, Hkv=8, d=128, rotary=128,
             pairs="halves", norm=True, base=1000000.0, scaling="", lens=3),
        # the decode step over an e4m3 cache: most tiles hold keys already
        dict(name="step8_decode", kind="step8", B=64, most_new=1, longest=4000, page=128, Hq=32, Hkv=8, d=128, rotary=128,
             pairs="halves", norm=False, base=500000.0, scaling="", lens=2),
        # the prefill chunks over an e4m3 cache
        dict(name="step8_prefill", kind="step8", B=9, most_new=6000, longest=9000, page=64, Hq=32, Hkv=8, d=128, rotary=128,
             pairs="halves", norm=False, base=500000.0, scaling="bands", lens=3),
        # one request of a conversation is taken out of its pages
        dict(name="read_one", kind="read", B=1, longest=3000, page=16, Hkv=8, d=128, lens=1),
        # the cached prefixes of a batch
        dict(name="read8_batch", kind="read8", B=16, longest=16000, page=128, Hkv=8, d=128, lens=5),
        # short chunks of a few conversations behind their histories
        dict(name="prefill8_short", kind="prefill8", B=4, most_new=130, longest=6000, page=64, Hq=32, Hkv=8, d=128, lens=4),
        # a long prompt's chunk behind what it has cached so far
        dict(name="prefill8_long", kind="prefill8", B=1, most_new=2048, longest=30000, page=128, Hq=32, Hkv=8, d=128, lens=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["train", "train", "packed", "rotate", "step", "step", "step8", "step8", "read", "read8", "prefill8"])
    c = dict(kind=kind)
    if kind in ("train", "packed", "rotate", "step", "step8"):
        heads = rng.choice([(2, 2), (8, 2), (16, 4), (16, 16), (32, 8)])
        d = rng.choice([64, 128, 128] if kind == "step8" else [64, 80, 96, 128, 128, 256])
        c.update(Hq=heads[0], Hkv=heads[1], d=d, rotary=rng.choice([d, d, d // 2, d // 4]), pairs=rng.choice(["halves", "halves", "neighbours"]),
                 norm=rng.random() < 0.4, base=rng.choice([10000.0, 500000.0]), scaling=rng.choice(["", "", "linear", "ntk", "yarn", "bands"]))
    if kind in ("train", "rotate"):
        n = _log(rng, 10, 32768)
        c.update(B=max(1, min(rng.choice([1, 2, 8]), 32768 // n)), N=n, start=rng.choice([0, 0, _log(rng, 10, 1000000)]))
    elif kind == "packed":
        c.update(seqs=rng.randint(2, 12), longest=_log(rng, 100, 2500), lens=rng.randrange(1000))
    elif kind in ("step", "step8"):
        small = rng.random() < 0.5
        c.update(B=_log(rng, 1, 64) if small else _log(rng, 1, 9), most_new=rng.choice([1, 1, 4]) if small else _log(rng, 50, 6000),
                 longest=_log(rng, 200, 9000), page=rng.choice([16, 64, 128, 256]), lens=rng.randrange(1000))
    elif kind in ("read", "read8"):
        c.update(B=_log(rng, 1, 32), longest=_log(rng, 100, 16000), page=rng.choice([16, 64, 128, 256]), Hkv=rng.choice([1, 2, 8]),
                 d=rng.choice([64, 128, 128]), lens=rng.randrange(1000))
    else:
        heads = rng.choice([(8, 2), (16, 16), (32, 8)])
        new = _log(rng, 20, 2000)
        c.update(B=max(1, min(rng.choice([1, 2, 4, 8]), 2048 // new)), most_new=new, longest=_log(rng, 100, 30000 if new > 500 else 8000),
                 page=rng.choice([16, 64, 128, 256]), Hq=heads[0], Hkv=heads[1], d=rng.choice([64, 128, 128]), lens=rng.randrange(1000))
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
    """(keys that each request holds, its new tokens) of a case over a cache."""
    r = random.Random(case["lens"] * 7 + 1)
    held = [r.randint(0, case["longest"]) for _ in range(case["B"])]
    if case["kind"] == "prefill8":
        held[0] = case["longest"]
    if case["most_new"] > 8:
        new = [r.randint(1, case["most_new"]) for _ in range(case["B"])]
        new[0] = case["most_new"]
    else:
        new = [case["most_new"]] * case["B"]
    return held, new


def work(case):
    kind = case["kind"]
    if kind in ("read", "read8"):
        n = 2 * sum(_lengths(case["B"], case["longest"], case["lens"])) * case["Hkv"] * case["d"]
        return {"bytes": n * (4 if kind == "read" else 3), "flops": 0 if kind == "read" else n}
    if kind == "prefill8":
        held, new = _serving(case)
        keys, pairs = sum(h + n for h, n in zip(held, new)), sum(n * h + n * (n + 1) // 2 for h, n in zip(held, new))
        return {"bytes": 2 * keys * case["Hkv"] * case["d"] + sum(new) * case["Hq"] * (4 * case["d"] + 4), "flops": 4 * pairs * case["Hq"] * case["d"]}
    if kind in ("step", "step8"):
        rows = sum(_serving(case)[1])
        q, kv = rows * case["Hq"] * case["d"], rows * case["Hkv"] * case["d"]
        return {"bytes": 4 * q + 2 * kv * (4 if kind == "step" else 3) + 12 * rows, "flops": 3 * (q + kv)}
    rows = sum(_lengths(case["seqs"], case["longest"], case["lens"])) if kind == "packed" else case["B"] * case["N"]
    n = rows * (case["Hq"] + case["Hkv"]) * case["d"]
    if kind == "rotate":
        return {"bytes": 4 * n, "flops": 3 * n}
    return {"bytes": 8 * n, "flops": 6 * n}      # q, k and the incoming gradients in; the rotated ones and the gradients out


# ------------------------------------------------------------------------------------------------ inputs

def _frequencies(case):
    """(radians per position of each pair in 64 bits, factor on the rotated columns) for the case's scaling."""
    R, base = case["rotary"], case["base"]
    i = torch.arange(R // 2, dtype=torch.float64)
    f = base ** (-2 * i / R)
    how, by, before = case["scaling"], 8.0, 8192
    if how == "linear":
        f = f / by
    elif how == "ntk":
        f = (base * by ** (R / (R - 2))) ** (-2 * i / R)
    elif how == "yarn":          # pairs that turn 32 times and more within the first length stay, those below one turn are stretched
        at = [R * math.log(before / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (32, 1)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), R - 1)
        ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        return f / by * ramp + f * (1 - ramp), 0.1 * math.log(by) + 1
    elif how == "bands":         # by wavelength: up to a quarter of the first length as they are, beyond it stretched
        part = ((before * f / (2 * math.pi) - 1) / 3).clamp(0, 1)
        f = f / by * (1 - part) + f * part
    return f, 1.0


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    kind = case["kind"]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=dev).to(torch.bfloat16)

    def codes(*shape):
        return (torch.randn(shape, generator=gen, device=dev) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)

    s = dict(case=case)
    if "rotary" in case:
        f, s["magnitude"] = _frequencies(case)
        s["f"] = f.to(dev)
        s["wq"], s["wk"] = (randn(case["d"]) * 0.2 + 1 for _ in range(2)) if case["norm"] else (None, None)
    if kind in ("train", "packed", "rotate"):
        if kind == "packed":
            lens = _lengths(case["seqs"], case["longest"], case["lens"])
            s["cu"] = torch.tensor([0] + lens, device=dev).cumsum(0).to(torch.int32)
            B, N = 1, sum(lens)
        else:
            B, N = case["B"], case["N"]
            s["positions"] = None
            if case["start"]:
                s["positions"] = (torch.randint(0, case["start"], (B, 1), generator=gen, device=dev) + torch.arange(N, device=dev)).to(torch.int32)
        # q and k as parts of one projection's output
        x = randn(B, N, case["Hq"] + 2 * case["Hkv"], case["d"])
        s["q"], s["k"] = x[:, :, :case["Hq"]], x[:, :, case["Hq"]:case["Hq"] + case["Hkv"]]
        if kind != "rotate":
            s["dq"], s["dk"] = randn(B, N, case["Hq"], case["d"]), randn(B, N, case["Hkv"], case["d"])
        return s
    ps, B, Hkv, d = case["page"], case["B"], case["Hkv"], case["d"]
    held, new = (_lengths(B, case["longest"], case["lens"]), [0] * B) if kind in ("read", "read8") else _serving(case)
    grown, total = [-(-(h + n) // ps) for h, n in zip(held, new)], sum(new)
    pool = sum(grown) + 5
    order = torch.randperm(pool, generator=gen, device=dev).to(torch.int32)      # the pages of a request lie anywhere in the pool
    page = (pool, ps, Hkv, d)
    h, n = torch.tensor(held, device=dev), torch.tensor(new, device=dev)
    if kind in ("read", "read8", "prefill8"):
        first = torch.tensor([0] + grown, device=dev).cumsum(0)[:-1]
        x = torch.arange(max(grown), device=dev)[None]
        mine = x < torch.tensor(grown, device=dev)[:, None]
        s["block_table"] = torch.where(mine, order[(first[:, None] + x).clamp(max=pool - 1)], torch.full_like(order[:1], -1))
        s["seqlens"], s["rows"] = (h + n).to(torch.int32), sum(held) + total
        s["cu"] = torch.nn.functional.pad((h + n).cumsum(0), (1, 0)).to(torch.int32)
        if kind == "prefill8":
            s["q"], s["longest"], s["scale"] = randn(1, total, case["Hq"], d), max(new), 1 / math.sqrt(d)
            s["cu_q"] = torch.nn.functional.pad(n.cumsum(0), (1, 0)).to(torch.int32)
        for x in ("k", "v"):
            s[x + "pages"] = randn(*page) if kind == "read" else codes(*page)
            if kind != "read":
                s[x + "scale"] = torch.rand((pool, Hkv, max(1, ps // 128)), generator=gen, device=dev) * 0.01 + 0.005
        return s
    # slots of the new rows, request by request, behind the keys that it holds; the last request has no place (slot -1)
    first = torch.tensor([0] + grown, device=dev).cumsum(0)[:-1]
    seq = torch.repeat_interleave(torch.arange(B, device=dev), n, output_size=total)
    pos = h[seq] + torch.arange(total, device=dev) - (n.cumsum(0) - n)[seq]
    slots = order[first[seq] + pos // ps].to(torch.int64) * ps + pos % ps
    if B > 1:
        slots = torch.where(seq == B - 1, torch.full_like(slots, -1), slots)
    s["slots"], s["positions"] = slots, pos.to(torch.int32)
    x = randn(total, case["Hq"] + 2 * Hkv, d)
    if kind == "step8" and not case["norm"]:     # a tenth of the rows are larger than what their tile holds
        x = torch.where(torch.rand((total, 1, 1), generator=gen, device=dev) < 0.1, x * 4, x)
    s["q"], s["k"], s["v"] = x.split([case["Hq"], Hkv, Hkv], 1)
    for x in ("k", "v"):
        s[x + "pages"] = randn(*page) if kind == "step" else codes(*page)
        if kind == "step8":
            s[x + "scale"] = torch.rand((pool, Hkv, max(1, ps // 128)), generator=gen, device=dev) * 0.01 + 0.005
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind in ("train", "packed", "rotate"):
        return _train(state)
    return {"step": _step, "step8": _step, "read": _read, "read8": _read, "prefill8": _prefill8}[kind](state)


def _own(s):
    from paper_2609_32712_b200 import mala
    c, kind = s["case"], s["case"]["kind"]
    if "rotary" in c:
        rot = mala.Rotary(s["f"], interleaved=c["pairs"] == "neighbours", magnitude=s["magnitude"])
        norm = mala.HeadNorm(s["wq"], s["wk"], EPS) if c["norm"] else None
    if kind in ("train", "rotate"):
        q, k = mala.rotary(s["q"], s["k"], rot, positions=s["positions"], norm=norm)
        if kind == "rotate":
            return q, k
        return (q, k) + mala.rotary_bwd(s["dq"], s["dk"], rot, positions=s["positions"], norm=norm, q=s["q"], k=s["k"])
    if kind == "packed":
        q, k = mala.rotary_varlen(s["q"], s["k"], s["cu"], s["cu"], rot, norm=norm)
        return (q, k) + mala.rotary_varlen_bwd(s["dq"], s["dk"], s["cu"], s["cu"], rot, norm=norm, q=s["q"], k=s["k"])
    if kind == "step":
        q = mala.rotary_write(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["kpages"], s["vpages"], rot, norm=norm)
        return q, s["kpages"], s["vpages"]
    if kind == "step8":
        q = mala.rotary_write_fp8(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["kpages"], s["vpages"], s["kscale"], s["vscale"], rot, norm=norm)
        return q, s["kpages"], s["kscale"], s["vpages"], s["vscale"]
    if kind == "read":
        return mala.cache_read(s["kpages"], s["vpages"], s["block_table"], s["seqlens"], s["rows"])
    if kind == "read8":
        return mala.cache_read_fp8(s["kpages"], s["vpages"], s["kscale"], s["vscale"], s["block_table"], s["seqlens"], s["rows"])
    return mala.fwd_paged_fp8(s["q"], s["kpages"], s["vpages"], s["kscale"], s["vscale"], s["cu_q"], s["block_table"], s["seqlens"], s["longest"],
                              s["rows"], s["scale"], 0.0)[:2]


def _angles(s, pos):
    """(cos, sin) [..., R/2] at whole positions: the angles in 64 bits."""
    a = pos.double()[..., None] * s["f"]
    return a.cos().float() * s["magnitude"], a.sin().float() * s["magnitude"]


def _turn(y, cos, sin, c):
    """y [..., H, d] in 32 bits with its first R columns turned; cos, sin [..., 1, R/2]."""
    R = c["rotary"]
    y1, y2 = (y[..., :R // 2], y[..., R // 2:R]) if c["pairs"] == "halves" else (y[..., 0:R:2], y[..., 1:R:2])
    z1, z2 = y1 * cos - y2 * sin, y2 * cos + y1 * sin
    z = torch.cat([z1, z2], -1) if c["pairs"] == "halves" else torch.stack([z1, z2], -1).flatten(-2)
    return torch.cat([z, y[..., R:]], -1)


def _normed(x, w):
    x = x.float()
    return x if w is None else x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * w.float()


def _train(s):
    c = s["case"]
    if c["kind"] == "packed":
        row = torch.arange(s["q"].shape[1], device=s["q"].device)
        cu = s["cu"].long()
        pos = (row - cu[torch.searchsorted(cu[1:], row, right=True)])[None]
    else:
        pos = torch.arange(c["N"], device=s["q"].device)[None] if s["positions"] is None else s["positions"]
    cos, sin = (t[:, :, None] for t in _angles(s, pos))
    out = tuple(_turn(_normed(s[x], s["w" + x]), cos, sin, c).to(torch.bfloat16) for x in ("q", "k"))
    if c["kind"] == "rotate":
        return out
    (dq, dwq), (dk, dwk) = (_train_back(s[x], s["d" + x], s["w" + x], cos, sin, c) for x in ("q", "k"))
    return *out, dq, dk, dwq, dwk


def _train_back(x, dy, w, cos, sin, c):
    g = _turn(dy.float(), cos, -sin, c)
    if w is None:
        return g.to(torch.bfloat16), None
    x = x.float()
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    n, gw = x * r, g * w.float()
    dx = r * (gw - n * (gw * n).mean(-1, keepdim=True))
    return dx.to(torch.bfloat16), (g * n).sum((0, 1, 2), dtype=torch.float64).float()


def _step(s):
    c = s["case"]
    cos, sin = (t[:, None] for t in _angles(s, s["positions"]))
    q = _turn(_normed(s["q"], s["wq"]), cos, sin, c).to(torch.bfloat16)
    k, v = _turn(_normed(s["k"], s["wk"]), cos, sin, c), s["v"].float()
    ok = s["slots"] >= 0
    at = s["slots"][ok]
    if c["kind"] == "step":
        s["kpages"].view(-1, *k.shape[1:])[at] = k[ok].to(torch.bfloat16)
        s["vpages"].view(-1, *v.shape[1:])[at] = v[ok].to(torch.bfloat16)
        return q, s["kpages"], s["vpages"]
    unit = min(c["page"], 128)
    units, back = torch.unique(at // unit, return_inverse=True)      # the tiles (or pages) that get new keys
    new = torch.zeros((units.numel(), unit), device=at.device, dtype=torch.bool)
    new[back, at % unit] = True
    held = torch.arange(unit, device=at.device)[None] < new.long().argmax(1)[:, None]   # keys there before
    return (q, *_step8_one(k[ok], s["kpages"], s["kscale"], at, units, back, new, held),
            *_step8_one(v[ok], s["vpages"], s["vscale"], at, units, back, new, held))


def _step8_one(x, pages, scale, at, units, back, new, held):
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


def _values(s, x, pages):
    """Keys or values of the pages of a block table's entries in 32 bits: [..., page size, Hkv, d]."""
    t = s[x + "pages"][pages].float()
    if x + "scale" not in s:
        return t
    ps = t.shape[-3]
    scale = s[x + "scale"][pages].transpose(-1, -2)                  # [..., units of a page, Hkv]
    return t * scale.repeat_interleave(ps // scale.shape[-2], -2)[..., None]


def _read(s):
    ps, cu = s["case"]["page"], s["cu"].long()
    row = torch.arange(s["rows"], device=cu.device)
    seq = torch.searchsorted(cu[1:], row, right=True)
    pos = row - cu[seq]
    page, at = s["block_table"][seq, pos // ps].long(), pos % ps
    out = []
    if s["case"]["kind"] == "read":
        out = [s["kpages"][page, at], s["vpages"][page, at]]
    else:
        unit = min(ps, 128)
        out = [(s[x + "pages"].view(torch.uint8)[page, at].view(torch.float8_e4m3fn).float() * s[x + "scale"][page, :, at // unit][..., None]).to(torch.bfloat16)
               for x in ("k", "v")]
    return out[0][None], out[1][None], s["cu"]


def _prefill8(s):
    c = s["case"]
    cu, nk = s["cu_q"].long(), s["seqlens"].long()
    nq, M, G, d, dev = cu[1:] - cu[:-1], s["longest"], c["Hq"] // c["Hkv"], c["d"], s["q"].device
    pages = s["block_table"].long().clamp(min=0)
    k, v = (_values(s, x, pages).flatten(1, 2).permute(0, 2, 1, 3) for x in ("k", "v"))      # [B, Hkv, keys, d]
    x = torch.arange(M, device=dev)
    q = s["q"][0][(cu[:-1, None] + x).clamp(max=s["q"].shape[1] - 1)].float()                # one padded row per request
    q = q.view(c["B"], M, c["Hkv"], G, d).permute(0, 2, 3, 1, 4).reshape(c["B"], c["Hkv"], G * M, d)
    seen = (nk - nq)[:, None] + x                                                            # last key that a query sees
    hidden = torch.arange(k.shape[2], device=dev)[None, None] > seen[:, :, None]
    z = (q @ k.transpose(-1, -2)).mul_(s["scale"]).view(c["B"], c["Hkv"], G, M, -1)
    z.masked_fill_(hidden[:, None, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    p = z.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = (p.view(c["B"], c["Hkv"], G * M, -1) @ v).view(c["B"], c["Hkv"], G, M, d) / l
    row = torch.arange(s["q"].shape[1], device=dev)
    seq = torch.searchsorted(cu[1:], row, right=True)
    o = o.permute(0, 3, 1, 2, 4).reshape(c["B"], M, c["Hq"], d)[seq, row - cu[seq]]
    lse = (m + l.log())[..., 0].reshape(c["B"], c["Hq"], M).permute(1, 0, 2)[:, seq, row - cu[seq]]
    return o[None].to(torch.bfloat16), lse


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("train", "packed", "rotate"):
        return _exact_train(s)
    if kind in ("step", "step8"):
        return _exact_step(s)
    if kind == "prefill8":
        return _exact_prefill8(s)
    k, v = (torch.cat(t)[None] for t in zip(*(_exact_request(s, b) for b in range(case["B"]))))
    return k, v, None        # (offsets are whole numbers)


def _exact_rotation(s, pos):
    """The rotations of rows at `pos` as complex numbers of modulus `magnitude`, [..., R/2]."""
    return torch.polar(torch.full((), s["magnitude"], dtype=torch.float64, device=s["f"].device).expand(*pos.shape, s["f"].numel()).contiguous(),
                       pos.double()[..., None] * s["f"])


def _exact_turn(x, by, c):
    """x [..., H, d] times the complex numbers `by` [..., R/2], column by column."""
    R, x = c["rotary"], x.double()
    a = torch.arange(R // 2, device=x.device) * (1 if c["pairs"] == "halves" else 2)
    b = a + (R // 2 if c["pairs"] == "halves" else 1)
    z = torch.complex(x[..., a], x[..., b]) * by[..., None, :]
    out = x.clone()
    out[..., a], out[..., b] = z.real, z.imag
    return out


def _exact_train(s):
    c = s["case"]
    if c["kind"] == "packed":
        pos = torch.cat([torch.arange(b - a) for a, b in zip(s["cu"].tolist(), s["cu"].tolist()[1:])])[None].to(s["q"].device)
    else:
        pos = s["positions"] if s["positions"] is not None else torch.arange(c["N"], device=s["q"].device).expand(c["B"], -1)
    out, grads, dws = [], [], []
    for x in ("q", "k"):
        w = None if s["w" + x] is None else s["w" + x].double()
        y, dx, dw = [], [], torch.zeros(c["d"], device=s["q"].device, dtype=torch.float64)
        for b in range(s["q"].shape[0]):
            t, by = s[x][b].double(), _exact_rotation(s, pos[b])
            scale = torch.ones((), device=t.device, dtype=torch.float64)
            if w is not None:
                scale = 1 / torch.sqrt((t * t).sum(-1, keepdim=True) / c["d"] + EPS)
            y.append(_exact_turn(t * scale * (1 if w is None else w), by, c))
            if c["kind"] == "rotate":
                continue
            g = _exact_turn(s["d" + x][b], by.conj(), c)
            if w is not None:
                dw += torch.einsum("nhd,nhd->d", g, t * scale)
                g = g * w
                g = scale * g - t * scale ** 3 * (g * t).sum(-1, keepdim=True) / c["d"]
            dx.append(g)
        out.append(torch.stack(y))
        if c["kind"] != "rotate":
            grads.append(torch.stack(dx))
            dws.append(None if w is None else dw)
    return (*out, *grads, *dws)


def _exact_step(s):
    """Codes before their rounding to 8 bits, and scales."""
    c = s["case"]
    by = _exact_rotation(s, s["positions"])
    rows = {}
    for x in ("q", "k"):
        t = s[x].double()
        if c["norm"]:
            t = t / torch.sqrt((t * t).sum(-1, keepdim=True) / c["d"] + EPS) * s["w" + x].double()
        rows[x] = _exact_turn(t, by, c)
    rows["v"] = s["v"].double()
    P, ps, H, d = s["kpages"].shape
    slots, dev = s["slots"], s["slots"].device
    have = torch.nonzero(slots >= 0)[:, 0]
    out = [rows["q"]]
    for x in ("k", "v"):
        flat = s[x + "pages"].double().view(-1, H, d)
        if c["kind"] == "step":
            out.append(flat.index_copy(0, slots[have], rows[x][have]).view(P, ps, H, d))
            continue
        unit = min(ps, 128)
        u, back = torch.unique(slots[have] // unit, return_inverse=True)
        least = torch.full((u.numel(),), unit, device=dev).scatter_reduce(0, back, slots[have] % unit, "amin")
        a = torch.zeros((u.numel(), H), device=dev, dtype=torch.float64)
        a.scatter_reduce_(0, back[:, None].expand(-1, H), rows[x][have].abs().amax(2) / 448, "amax")
        old = s[x + "scale"].double().permute(0, 2, 1).reshape(-1, H)
        now = torch.where((least == 0)[:, None], torch.where(a > 0, a, 1.0), torch.maximum(a, old[u]))
        ratio = torch.where(least[:, None] > 0, old[u] / now, 1.0)
        kept = (torch.arange(unit, device=dev)[None] < least[:, None])[:, :, None, None]
        units = flat.view(-1, unit, H, d)
        units[u] = torch.where(kept, units[u] * ratio[:, None, :, None], units[u])
        flat[slots[have]] = rows[x][have] / now[back][:, :, None]
        scales = old.clone()
        scales[u] = now
        out += [flat.view(P, ps, H, d), scales.view(P, -1, H).permute(0, 2, 1).contiguous()]
    return tuple(out)


def _exact_request(s, b):
    """Keys and values of request b in 64 bits, [keys, Hkv, d]."""
    n, ps = int(s["seqlens"][b]), s["case"]["page"]
    pages = s["block_table"][b, :-(-n // ps)].long()
    out = []
    for x in ("k", "v"):
        t = s[x + "pages"][pages].double()
        if x + "scale" in s:
            per = s[x + "scale"].shape[2]
            t = (t.view(len(pages), per, ps // per, *t.shape[2:]) * s[x + "scale"][pages].double().permute(0, 2, 1)[:, :, None, :, None]).flatten(1, 2)
        out.append(t.flatten(0, 1)[:n])
    return out


def _exact_prefill8(s):
    c = s["case"]
    G, cu = c["Hq"] // c["Hkv"], s["cu_q"].tolist()
    o = torch.zeros_like(s["q"], dtype=torch.float64)
    lse = torch.zeros((c["Hq"], o.shape[1]), device=o.device, dtype=torch.float64)
    for b in range(c["B"]):
        k, v = _exact_request(s, b)
        rows = slice(cu[b], cu[b + 1])
        nq, nk = cu[b + 1] - cu[b], k.shape[0]
        mask = torch.ones((nq, nk), device=o.device, dtype=torch.bool).tril(nk - nq)
        for h in range(c["Hq"]):
            x = (s["q"][0, rows, h].double() @ k[:, h // G].T * s["scale"]).where(mask, -math.inf)
            lse[h, rows] = torch.logsumexp(x, 1)
            o[0, rows, h] = torch.exp(x - lse[h, rows][:, None]) @ v[:, h // G]
    return o, lse
