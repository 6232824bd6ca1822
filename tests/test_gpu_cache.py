"""Block tables, slots, the release of pages and the writes into bf16 and e4m3 pages, against plain implementations; and a serving
run of all of them with the paged attention calls."""
import math
import random

import numpy as np
import pytest
import torch

from tests import bias_reference as R
from tests import parity

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mala():
    from paper_2609_32712_b200 import mala as m
    m.lib()
    return m


def _randn(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pool:
    """The same bookkeeping in plain Python."""

    def __init__(self, lens, width, ps, num_pages, seed):
        r = random.Random(seed)
        self.free = list(range(num_pages))
        r.shuffle(self.free)
        self.ps, self.width, self.num_pages = ps, width, num_pages
        self.lens = list(lens)
        self.table = [[-1] * width for _ in lens]
        for b, n in enumerate(lens):
            for x in range(-(-n // ps)):
                self.table[b][x] = self.free.pop()

    def device(self):
        free = _i32(self.free + [-7] * (self.num_pages - len(self.free)))
        return _i32(self.lens), _i32(self.table), free, _i32([len(self.free)])

    def add(self, new):
        cu, slots, free, left, upto = [0], [], list(self.free), len(self.free), 0
        for b, n in enumerate(new):
            n = max(n, 0)
            cu.append(cu[-1] + n)
            have = -(-self.lens[b] // self.ps)
            fits = self.lens[b] + n <= self.width * self.ps
            need = -(-(self.lens[b] + n) // self.ps) - have if fits else 0
            upto += need
            if not fits or (need and upto > len(free)):
                slots += [-1] * n
                continue
            for x in range(need):
                self.table[b][have + x] = self.free.pop()
            slots += [self.table[b][p // self.ps] * self.ps + p % self.ps for p in range(self.lens[b], self.lens[b] + n)]
            self.lens[b] += n
        return cu, slots

    def release(self, done):
        for b, f in enumerate(done):
            if f:
                self.free += self.table[b][:-(-self.lens[b] // self.ps)]
                self.lens[b] = 0


@pytest.mark.parametrize("B,longest,most,ps,width,spare", [
    (1, 0, 1, 16, 4, 3), (1, 100, 0, 16, 8, 0), (5, 40, 30, 8, 12, 40), (64, 400, 1, 16, 40, 100), (33, 300, 700, 128, 6, 60),
    (33, 300, 700, 128, 10, 20), (1000, 50, 20, 64, 3, 400), (1025, 20, 3, 8, 5, 2000), (5000, 30, 2, 32, 3, 3000), (3, 500, 9000, 256, 40, 200),
    (16384, 10, 1, 16, 2, 20000)])
def test_tables_and_release(mala, B, longest, most, ps, width, spare):
    """Several steps in a row: lengths with a refused request and an exhausted pool among them, rows behind the last request."""
    r = random.Random(B * 31 + most)
    lens = [r.randint(0, min(longest, width * ps)) for _ in range(B)]
    pool = Pool(lens, width, ps, sum(-(-n // ps) for n in lens) + spare, B)
    for step in range(3):
        seqlens, table, free, count = pool.device()
        done = [r.random() < 0.2 for _ in range(B)] if step else [False] * B
        held, count2 = mala.release_pages(torch.tensor(done, device="cuda"), seqlens, table, free, count, ps)
        pool.release(done)
        assert held.tolist() == pool.lens and count2.item() == len(pool.free) and free.tolist()[:len(pool.free)] == pool.free
        new = [r.randint(-1 if most > 2 else 0, most) for _ in range(B)]
        extra = r.choice([0, 5])
        total = sum(max(n, 0) for n in new)
        before = [list(t) for t in table.tolist()]
        cu, lens2, slots, left = mala.page_tables(held, _i32(new), table, free, count2, ps, total + extra)
        old = list(pool.lens)
        wcu, wslots = pool.add(new)
        assert cu.tolist() == wcu and lens2.tolist() == pool.lens and left.item() == len(pool.free)
        assert slots.tolist() == wslots + [-1] * extra
        got = table.tolist()
        for b in range(B):
            n = -(-pool.lens[b] // ps)
            assert got[b][:n] == pool.table[b][:n]
            assert got[b][n:] == before[b][n:]         # (what is not given out stays as it was)
            assert pool.lens[b] >= old[b]
    short = mala.page_tables(held, _i32(new), table, free, count2, ps, max(total // 2, 0))[2]     # (fewer slots than tokens)
    assert short.tolist() == wslots[:total // 2]


def test_slots_beyond_32_bits(mala):
    """Pages so far out that their slots pass 2^31."""
    ps, far = 1024, 3_000_000
    table = _i32([[far, -1, -1]])
    free = torch.arange(far - 1, far + 3, dtype=torch.int32, device="cuda")
    cu, lens, slots, left = mala.page_tables(_i32([1000]), _i32([1500]), table, free, _i32([4]), ps, 1500)
    want = [far * ps + 1000 + x for x in range(24)] + [(far + 2) * ps + x for x in range(1024)] + [(far + 1) * ps + x for x in range(452)]
    assert slots.tolist() == want and lens.item() == 2500 and left.item() == 2


def test_pages_beyond_32_bits(mala):
    """Pages of which the last ones begin behind 2^32 bytes, in a call that writes the first and the last one, bf16 and e4m3."""
    for item, ps, Hkv, d in ((2, 128, 8, 128), (1, 128, 8, 128)):
        num = (1 << 32) // (ps * Hkv * d * item) + 3
        pages = [torch.empty((num, ps, Hkv, d), dtype=torch.bfloat16 if item == 2 else torch.float8_e4m3fn, device="cuda") for _ in range(2)]
        slots = torch.cat([torch.arange(ps), torch.arange(ps) + (num - 1) * ps]).cuda()
        g = torch.Generator(device="cuda").manual_seed(7)
        k, v = (torch.randn((2 * ps, Hkv, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        if item == 2:
            mala.cache_write(k, v, slots, *pages)
            for x, p in zip((k, v), pages):
                assert torch.equal(p[0], x[:ps]) and torch.equal(p[-1], x[ps:])
        else:
            scales = [torch.zeros((num, Hkv, 1), device="cuda") for _ in range(2)]
            mala.cache_write_fp8(k, v, slots, *pages, *scales)
            for x, p, s in zip((k, v), pages, scales):
                for at, rows in ((0, x[:ps]), (num - 1, x[ps:])):
                    want = rows.abs().amax((0, 2)).float() / torch.full((Hkv,), 448., device="cuda")
                    assert torch.equal(s[at, :, 0], want)
                    err = (p[at].float() * want[:, None] - rows.float()).abs()
                    assert (err <= 2.0 ** -4 * rows.float().abs() + 2.0 ** -10 * want[:, None] * 1.01).all()
        del pages


def _slots(B, longest, most, ps, seed, num_extra=3):
    r = random.Random(seed)
    lens = [r.randint(0, longest) for _ in range(B)]
    new = [r.randint(0, most) if most > 4 else most for _ in range(B)]
    pool = Pool(lens, 10 ** 4, ps, sum(-(-(a + b) // ps) for a, b in zip(lens, new)) + num_extra, seed)
    _, slots = pool.add(new)
    return torch.tensor(slots, dtype=torch.int64, device="cuda"), pool.num_pages, lens, new


@pytest.mark.parametrize("B,longest,most,ps,Hkv,d", [(1, 0, 1, 16, 1, 8), (64, 400, 1, 16, 8, 128), (7, 500, 900, 64, 2, 40), (5, 300, 300, 128, 3, 256),
                                                     (3, 10, 2, 8, 1, 64), (2, 1000, 3000, 256, 8, 128)])
def test_write(mala, B, longest, most, ps, Hkv, d):
    slots, pages, _, _ = _slots(B, longest, most, ps, B + most)
    rows = slots.numel()
    if rows > 2:
        slots[1] = -1
        slots[2] = pages * ps + 5                    # (beyond the pool)
    x = _randn(1, rows, 2 * Hkv, d)
    k, v = x[:, :Hkv], x[:, Hkv:]                    # views of one projection
    kp, vp = _randn(2, pages, ps, Hkv, d), _randn(3, pages, Hkv, ps, d).transpose(1, 2)   # key-major and head-major pages
    wk, wv = kp.clone(), vp.contiguous().clone()
    ok = (slots >= 0) & (slots < pages * ps)
    wk.view(-1, Hkv, d)[slots[ok]] = k[ok]
    wv.view(-1, Hkv, d)[slots[ok]] = v[ok]
    mala.cache_write(k, v, slots, kp, vp)
    assert torch.equal(kp, wk) and torch.equal(vp, wv)


def _plain_write8(x, pages, scale, slots):
    """Unit by unit, in fp32 as the operator is defined (division and both roundings to nearest even)."""
    P, ps, H, d = pages.shape
    unit = min(ps, 128)
    codes, scale = pages.clone().view(-1, H, d), scale.clone()
    s = slots.tolist()
    t = 0
    while t < len(s):
        if s[t] < 0:
            t += 1
            continue
        n = 1
        while t + n < len(s) and s[t + n] == s[t] + n and (s[t] + n) // unit == s[t] // unit:
            n += 1
        at, off = s[t], s[t] % unit
        page, tile = at // ps, (at % ps) // 128
        rows = x[t:t + n].float()
        top = rows.abs().amax((0, 2))
        want = top / torch.full_like(top, 448.0)      # (by a tensor: by a number torch multiplies with its rounded reciprocal)
        old = scale[page, :, tile].clone()
        new = torch.where(want > 0, want, torch.ones_like(want)) if off == 0 else torch.maximum(old, want)
        scale[page, :, tile] = new
        if off:
            held = codes[at - off:at].float()
            codes[at - off:at] = torch.where((new > old)[None, :, None], (held * old[None, :, None] / new[None, :, None]).clamp(-448, 448),
                                             held).to(torch.float8_e4m3fn)
        codes[at:at + n] = (rows / new[None, :, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
        t += n
    return codes.view(pages.shape), scale


@pytest.mark.parametrize("B,longest,most,ps,Hkv,d", [(1, 0, 1, 16, 1, 16), (64, 400, 1, 128, 4, 128), (40, 100, 3, 16, 2, 64), (7, 500, 900, 64, 2, 48),
                                                     (5, 300, 300, 128, 3, 128), (3, 1000, 2000, 256, 2, 128), (9, 300, 77, 32, 1, 112)])
def test_write_fp8(mala, B, longest, most, ps, Hkv, d):
    slots, pages, _, new = _slots(B, longest, most, ps, 5 * B + most)
    rows = slots.numel()
    if B > 1:
        slots[rows - new[-1]:] = -1                  # a request without places (the rows of a unit are neighbours: not one row of many)
    g = torch.Generator(device="cuda")
    g.manual_seed(B)
    big = torch.rand((rows, 1, 1), generator=g, device="cuda") < 0.2
    x = _randn(4, rows, 2 * Hkv, d)
    x = torch.where(big, x * 8, x)
    if rows > 3:
        x[3] = 0
    k, v = x[:, :Hkv], x[:, Hkv:]
    kp, vp = ((torch.randn((pages, ps, Hkv, d), generator=g, device="cuda") * 100).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.rand((pages, Hkv, max(1, ps // 128)), generator=g, device="cuda") * 0.01 + 0.004 for _ in range(2))
    want = [_plain_write8(a, b, c, slots) for a, b, c in ((k, kp, ks), (v, vp, vs))]
    mala.cache_write_fp8(k, v, slots, kp, vp, ks, vs)
    torch.cuda.synchronize()
    for (codes, scale), p, s in zip(want, (kp, vp), (ks, vs)):
        assert torch.equal(s, scale)
        assert torch.equal(p.view(torch.uint8), codes.view(torch.uint8))


def test_write_fp8_extremes(mala):
    """Units of zeros, of bf16's smallest and largest values, and every magnitude in between."""
    ps, d = 16, 16
    vals = torch.cat([torch.zeros(d), torch.full((d,), 2.0 ** -133), torch.full((d,), torch.finfo(torch.bfloat16).max), 2.0 ** torch.linspace(-120, 120, d),
                      torch.arange(1, d + 1).float() * 2.0 ** -130, -448 * torch.ones(d), torch.linspace(-3, 3, d)]).to(torch.bfloat16)
    x = vals.view(-1, 1, d).cuda().repeat_interleave(ps, 0)
    pages = x.shape[0] // ps
    slots = torch.arange(x.shape[0], device="cuda")
    kp = torch.zeros((pages, ps, 1, d), device="cuda").to(torch.float8_e4m3fn)
    vp, ks, vs = kp.clone(), torch.zeros((pages, 1, 1), device="cuda"), torch.zeros((pages, 1, 1), device="cuda")
    codes, scale = _plain_write8(x, kp, ks, slots)
    mala.cache_write_fp8(x, x, slots, kp, vp, ks, vs)
    assert torch.equal(ks, scale) and torch.equal(vs, scale)
    assert torch.equal(kp.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(kp.view(torch.uint8), vp.view(torch.uint8))


def test_a_call_without_rows(mala):
    kp = _randn(1, 2, 16, 1, 64)
    want = kp.clone()
    empty = kp.new_empty((0, 1, 64))
    mala.cache_write(empty, empty, torch.empty(0, dtype=torch.int64, device="cuda"), kp, kp.clone())
    assert torch.equal(kp, want)


@pytest.mark.parametrize("fp8", [False, True])
def test_a_serving_run(mala, fp8):
    """Requests arrive with prompts, are extended token by token, finish and make room for others: tables, writes and paged
    attention (with a bias where the cache is bf16) against attention over each request's own keys."""
    ps, Hq, Hkv, d, B, width = 64, 4, 2, 64, 6, 12
    num_pages = 30
    scale = 1 / math.sqrt(d)
    table = _randn(9, 32, Hq)
    bias = mala.RelativeBias(table)
    block_table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    free, count = torch.arange(num_pages, dtype=torch.int32, device="cuda"), _i32([num_pages])
    seqlens = _i32([0] * B)
    if fp8:
        kp, vp = (torch.zeros((num_pages, ps, Hkv, d), dtype=torch.uint8, device="cuda") for _ in range(2))
        ks, vs = (torch.ones((num_pages, Hkv, 1), device="cuda") for _ in range(2))
    else:
        kp, vp = (torch.zeros((num_pages, ps, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    keys = [torch.empty((0, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(B)]
    vals = [k.clone() for k in keys]
    r = random.Random(4)
    steps = [[300, 70, 1, 0, 500, 64]] + [[1] * B for _ in range(3)] + [[0, 200, 1, 130, 1, 1]] + [[1] * B for _ in range(2)]
    for step, new in enumerate(steps):
        done = [step == 4 and b in (0, 4) for b in range(B)]
        held, c2 = mala.release_pages(torch.tensor(done, device="cuda"), seqlens, block_table, free, count, ps)
        total = sum(new)
        cu, seqlens, slots, count = mala.page_tables(held, _i32(new), block_table, free, c2, ps, total)
        k, v, q = _randn(100 + step, total, Hkv, d), _randn(200 + step, total, Hkv, d), _randn(300 + step, 1, total, Hq, d)
        if fp8:
            mala.cache_write_fp8(k, v, slots, kp, vp, ks, vs)
        else:
            mala.cache_write(k, v, slots, kp, vp)
        assert (slots >= 0).all()
        at = 0
        for b, n in enumerate(new):
            if done[b]:
                keys[b], vals[b] = keys[b][:0], vals[b][:0]
            keys[b], vals[b] = torch.cat([keys[b], k[at:at + n]]), torch.cat([vals[b], v[at:at + n]])
            at += n
        assert seqlens.tolist() == [x.shape[0] for x in keys]
        if max(new) > 1:
            if fp8:
                continue
            o, _, _ = mala.fwd_paged(q, kp, vp, cu, block_table, seqlens, max(new), scale, 0.0)
            tab, got = torch.zeros_like(table), o[0]
        else:
            qd = q[0][:, None].contiguous()
            if fp8:
                o, _, _ = mala.decode_fp8_paged(qd, kp, vp, ks, vs, block_table, seqlens, scale, 0.0, 2)
                tab = torch.zeros_like(table)
            else:
                o, _, _ = mala.decode_paged_bias(qd, kp, vp, block_table, seqlens, bias, scale, 0.0, 2)
                tab = table
            got = o[:, 0]
        at = 0
        for b, n in enumerate(new):
            for h in range(Hq if n else 0):
                g = h // (Hq // Hkv)
                ref = R.head(q[0, at:at + n, h].double(), keys[b][:, g].double(), vals[b][:, g].double(), tab[:, h].double(), None, scale, 32, 128, False, True)
                err = (got[at:at + n, h].double() - ref["o"]).abs()
                if fp8:   # keys and values to e4m3, twice where a scale has grown: half a step each is 2^-4 of a value
                    assert (err.norm() / ref["o"].norm()).item() <= 2 * 2.0 ** -4
                else:
                    assert (err <= parity.BF16_U * (ref["o"].abs() + ref["a"]) * 1.02 + 1e-5).all()
            at += n
    assert mala.device_status() == 0


def test_captured_step(mala):
    """Tables and writes captured once, replayed on other lengths and rows."""
    ps, B, width, Hkv, d = 16, 8, 10, 2, 64
    pool = Pool([5, 0, 31, 32, 100, 16, 1, 70], width, ps, 60, 3)
    seqlens, table, free, count = pool.device()
    new = _i32([1] * B)
    k, v = _randn(1, B, Hkv, d), _randn(2, B, Hkv, d)
    kp, vp = _randn(3, 60, ps, Hkv, d), _randn(4, 60, ps, Hkv, d)

    def step():
        cu, lens, slots, left = mala.page_tables(seqlens, new, table, free, count, ps, B)
        mala.cache_write(k, v, slots, kp, vp)
        return lens, slots, left
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            lens, slots, left = step()
    for x in range(5):
        s0, t0, f0, c0 = pool.device()
        for a, b in ((seqlens, s0), (table, t0), (free, f0), (count, c0), (k, _randn(10 + x, B, Hkv, d)), (v, _randn(20 + x, B, Hkv, d))):
            a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        _, want = pool.add([1] * B)
        assert slots.tolist() == want and lens.tolist() == pool.lens and left.item() == len(pool.free)
        assert torch.equal(kp.view(-1, Hkv, d)[slots], k) and torch.equal(vp.view(-1, Hkv, d)[slots], v)


@pytest.mark.parametrize("new", [[2 ** 31 - 1, 5, 2 ** 31 - 1, 9, 1], [2 ** 31 - 1] * 5, [2 ** 30 + 7] * 4 + [3], [3, 2 ** 31 - 2, 2 ** 31 - 1, 3, 3]])
@pytest.mark.parametrize("rows", [40, 5000])
def test_more_rows_than_32_bits_count_stay_within_the_buffers(mala, new, rows):
    """The sum of new_tokens has to stay below 2^31.  Where it does not, table, list and slots are written nowhere else."""
    ps, width, B, pages = 16, 2 ** 31 // 16 // 2 ** 20 * 2 ** 10, 5, 64      # (a table of rows of 131072 entries)
    big = torch.full((B + 2, width), -3, dtype=torch.int32, device="cuda")
    table = big[1:-1]
    table[:, :3] = torch.arange(15, device="cuda", dtype=torch.int32).view(5, 3)
    free = torch.arange(20, 20 + pages, dtype=torch.int32, device="cuda")
    list_ = free.clone()
    cu, lens, slots, left = mala.page_tables(_i32([40, 33, 48, 1, 20]), _i32(new), table, list_, _i32([30]), ps, rows)
    torch.cuda.synchronize()
    assert (big[0] == -3).all() and (big[-1] == -3).all() and torch.equal(free, list_)
    given = table[:, 3:]
    assert ((given == -3) | ((given >= 20) & (given < 50))).all()
    assert (slots >= -1).all() and (slots < 50 * ps).all() and 0 <= left.item() <= 30


@pytest.mark.parametrize("ps,Hkv,d", [(128, 2, 128), (16, 4, 64), (256, 1, 48)])
def test_write_fp8_head_major_pages(mala, ps, Hkv, d):
    """Pages whose heads lie apart (a unit's rows of one head side by side), some rows to units that hold keys."""
    slots, pages, _, _ = _slots(5, 300, 200, ps, 77)
    rows = slots.numel()
    k, v = _randn(4, rows, Hkv, d) * 3, _randn(5, rows, Hkv, d)
    g = torch.Generator(device="cuda").manual_seed(6)
    kp, vp = ((torch.randn((pages, Hkv, ps, d), generator=g, device="cuda") * 100).clamp(-448, 448).to(torch.float8_e4m3fn).transpose(1, 2) for _ in range(2))
    ks, vs = (torch.rand((pages, Hkv, max(1, ps // 128)), generator=g, device="cuda") * 0.01 + 0.004 for _ in range(2))
    want = [_plain_write8(a, b.contiguous(), c, slots) for a, b, c in ((k, kp, ks), (v, vp, vs))]
    mala.cache_write_fp8(k, v, slots, kp, vp, ks, vs)
    for (codes, scale), p, s in zip(want, (kp, vp), (ks, vs)):
        assert torch.equal(s, scale)
        assert torch.equal(p.contiguous().view(torch.uint8), codes.view(torch.uint8))


@pytest.mark.parametrize("ps", [16, 128])
@pytest.mark.parametrize("grow", [False, True])
def test_a_unit_filled_token_by_token(mala, ps, grow):
    """What decode steps do: a unit's keys one call after the other.  Its scale ends as that of one call, and with n roundings after a key's own
    (one for each time the scale has grown since) the key is off by at most ((1 + 2^-4)^(n + 1) - 1) |x| + (n + 1) (1 + 2^-4)^n 2^-10 s: half
    a step of 2^-4 of the value or of 2^-10 of the scale each."""
    Hkv, d = 2, 64
    k, v = _randn(8, ps, Hkv, d), _randn(9, ps, Hkv, d)
    if grow:                                    # (a scale that grows with every key)
        k = (k.float() * 1.1 ** torch.arange(ps, device="cuda")[:, None, None]).to(torch.bfloat16)
    kp, vp = (torch.zeros((2, ps, Hkv, d), device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.full((2, Hkv, 1), 7.0, device="cuda") for _ in range(2))
    history = []
    for t in range(ps):
        mala.cache_write_fp8(k[t:t + 1], v[t:t + 1], torch.tensor([ps + t], device="cuda"), kp, vp, ks, vs)
        history.append((ks[1, :, 0].clone(), vs[1, :, 0].clone()))
    for x, p, s, i in ((k, kp, ks, 0), (v, vp, vs, 1)):
        scales = torch.stack([h[i] for h in history])                       # [ps, Hkv]
        top = x.float().abs().amax((0, 2))
        assert torch.equal(s[1, :, 0], top / torch.full_like(top, 448.0)) and (s[0] == 7).all()
        grown = (scales[1:] > scales[:-1]).double()
        n = torch.cat([grown.flip(0).cumsum(0).flip(0), torch.zeros_like(grown[:1])])[..., None]
        assert not grow or i or n.max() > ps // 3
        xd, f = x.double(), (1 + 2.0 ** -4) ** n
        bound = (f * (1 + 2.0 ** -4) - 1) * xd.abs() + (n + 1) * f * 2.0 ** -10 * s[1, :, 0].double()[None, :, None]
        err = (p[1].double() * s[1, :, 0].double()[None, :, None] - xd).abs()
        assert (err <= bound * (1 + 1e-5)).all()
