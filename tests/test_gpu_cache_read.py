"""Reads of a paged cache, bf16 and e4m3, and prompts over an e4m3 cache, against plain implementations; and a serving run in which tables, rotations,
writes, prompts and decode steps work together."""
import math

import pytest
import torch

from tests import parity
from tests import rotary_reference as R

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


def _cache(seed, fp8, lens, ps, Hkv, d, extra=2):
    per = [-(-n // ps) for n in lens]
    pool = sum(per) + 3
    order = torch.randperm(pool, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((len(lens), max(per) + extra), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    if fp8:
        pages = [(_randn(seed + x, pool, ps, Hkv, d).float() * 100).clamp(-448, 448).to(torch.float8_e4m3fn) for x in range(2)]
        scales = [_randn(seed + 2 + x, pool, Hkv, max(1, ps // 128)).float().abs() * 0.01 + 0.005 for x in range(2)]
    else:
        pages, scales = [_randn(seed + x, pool, ps, Hkv, d) for x in range(2)], []
    return pages, scales, table.cuda()


def _gather(pages, scale, table, lens, ps):
    """The same reads with torch: the values of each sequence's keys, rounded once to bf16."""
    out = []
    for b, n in enumerate(lens):
        x = torch.arange(n, device="cuda")
        page, at = table[b][x // ps].long(), x % ps
        if scale is None:
            out.append(pages[page, at])
        else:
            codes = pages.view(torch.uint8)[page, at].view(torch.float8_e4m3fn).float()
            out.append((codes * scale[page, :, at // 128][..., None]).to(torch.bfloat16))
    return torch.cat(out)


LENS = [[1], [300, 1, 0, 129, 16, 128], [5000, 17], [0, 0], [33] * 70]


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("ps,Hkv,d", [(16, 2, 128), (128, 3, 64), (64, 1, 96), (256, 8, 128), (32, 1, 16), (8, 2, 256), (128, 1, 80), (64, 5, 8)])
@pytest.mark.parametrize("fp8", [False, True])
def test_read(mala, lens, ps, Hkv, d, fp8):
    if fp8 and (ps == 8 or d % 16 or d > 128):
        ps, d = max(ps, 16), min(max(d // 16 * 16, 16), 128)
    (kp, vp), scales, table = _cache(3, fp8, lens, ps, Hkv, d)
    ks, vs = scales if fp8 else (None, None)
    total = sum(lens)
    for rows in (total, total + 300, total + 5):
        if rows == 0:
            continue
        junk = torch.full((1 << 16,), 3.0, device="cuda", dtype=torch.bfloat16)      # (what the allocator hands out next holds something)
        del junk
        k, v, cu = mala.cache_read_fp8(kp, vp, ks, vs, table, _i32(lens), rows) if fp8 else mala.cache_read(kp, vp, table, _i32(lens), rows)
        assert cu.tolist() == [sum(lens[:b]) for b in range(len(lens) + 1)] and k.shape == v.shape == (1, rows, Hkv, d)
        if total:
            assert torch.equal(k[0, :total], _gather(kp, ks, table, lens, ps)) and torch.equal(v[0, :total], _gather(vp, vs, table, lens, ps))
        assert (k[0, total:total + 128] == 0).all() and (v[0, total:total + 128] == 0).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_read_values_in_64_bits(mala, fp8):
    lens, ps, Hkv, d = [40, 150], 128 if fp8 else 16, 2, 64
    (kp, vp), scales, table = _cache(5, fp8, lens, ps, Hkv, d)
    out = mala.cache_read_fp8(kp, vp, *scales, table, _i32(lens), 190) if fp8 else mala.cache_read(kp, vp, table, _i32(lens), 190)
    for t, pages, s in zip(out, (kp, vp), scales or (None, None)):
        want = torch.cat([R.values(pages, s, table[b], n, ps) for b, n in enumerate(lens)])
        # a product rounded to fp32 (2^-24) and to bf16 (2^-8)
        assert ((t[0].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -23)).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_read_odd_calls(mala, fp8):
    """Rows behind the sequences stay as they were; too little room; lengths beyond the table and below 0; pages that are not there; views."""
    ps, Hkv, d = 64, 2, 64
    lens = [100, 70, 30]
    (kp, vp), scales, table = _cache(7, fp8, lens, ps, Hkv, d)
    L = mala.lib()

    def read(lens_, rows, k, v, cu, table_=table, B=3):
        views = (mala._view8(kp), mala._view8(vp), scales[0].data_ptr(), scales[1].data_ptr()) if fp8 else (mala._view(kp, mala._TIn), mala._view(vp, mala._TIn))
        f = L.mala_cache_read_fp8 if fp8 else L.mala_cache_read
        assert f(*views, table_.data_ptr(), lens_.data_ptr(), mala._view(k, mala._TOut), mala._view(v, mala._TOut), cu.data_ptr(), B, Hkv, kp.shape[0], ps,
                 table_.shape[1], rows, d, torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
    want = [_gather(p, s, table, lens, ps) for p, s in zip((kp, vp), scales or (None, None))]
    new = lambda rows: [torch.full((1, rows, Hkv, d), 5.0, device="cuda", dtype=torch.bfloat16) for _ in range(2)]  # noqa: E731
    cu = torch.full((6,), -9, dtype=torch.int32, device="cuda")
    k, v = new(700)
    read(_i32(lens), 600, k, v, cu)
    assert cu.tolist() == [0, 100, 170, 200, -9, -9]
    for t, w in zip((k, v), want):
        assert torch.equal(t[0, :200], w) and (t[0, 200:328] == 0).all() and (t[0, 328:] == 5).all()
    # too little room: what fits
    k, v = new(200)
    read(_i32(lens), 150, k, v, cu)
    assert cu.tolist()[:4] == [0, 100, 150, 150] and torch.equal(k[0, :150], want[0][:150]) and (k[0, 150:] == 5).all() and (v[0, 150:] == 5).all()
    # lengths beyond what the table's row maps count as that, below 0 as 0; entries that name no page give 0
    k, v = new(2000)
    read(_i32([2 ** 31 - 1, -5, 30]), 1000, k, v, cu)
    room = table.shape[1] * ps
    assert cu.tolist()[:4] == [0, room, room, room + 30]
    assert torch.equal(k[0, :100], want[0][:100]) and (k[0, 128:room] == 0).all() and torch.equal(v[0, room:room + 30], want[1][170:200])
    wrong = table.clone()
    wrong[0, 0], wrong[1, 0] = kp.shape[0], -2 ** 31
    k, v = new(300)
    read(_i32(lens), 200, k, v, cu, wrong)
    assert (k[0, :64] == 0).all() and torch.equal(k[0, 64:100], want[0][64:100]) and (v[0, 100:164] == 0).all() and torch.equal(v[0, 164:200], want[1][164:200])
    # head-major outputs
    wide = torch.zeros((Hkv, 200, 2 * d), device="cuda", dtype=torch.bfloat16)
    hk, hv = (wide[..., x * d:(x + 1) * d].transpose(0, 1)[None] for x in range(2))
    read(_i32(lens), 200, hk, hv, cu)
    assert torch.equal(hk[0], want[0]) and torch.equal(hv[0], want[1])
    # head-major pages
    hm = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (kp, vp)]
    got = mala.cache_read_fp8(*hm, *scales, table, _i32(lens), 200) if fp8 else mala.cache_read(*hm, table, _i32(lens), 200)
    assert torch.equal(got[0][0], want[0]) and torch.equal(got[1][0], want[1])


def test_read_behind_2_to_the_32_bytes(mala):
    ps, Hkv, d = 128, 1, 128
    pool = 2 ** 32 // (ps * d) + 8
    kp, vp = (torch.zeros((pool, ps, Hkv, d), dtype=torch.uint8, device="cuda") for _ in range(2))
    tail = (_randn(1, 3, ps, Hkv, d).float() * 50).to(torch.float8_e4m3fn)
    kp[-3:], vp[-3:] = tail.view(torch.uint8), tail.flip(0).view(torch.uint8)
    s = torch.rand((pool, Hkv, 1), device="cuda") + 0.5
    table = _i32([[pool - 1, pool - 3], [pool - 2, 0]])
    k, v, _ = mala.cache_read_fp8(kp, vp, s, s, table, _i32([200, 128]), 328)
    assert torch.equal(k[0], _gather(kp, s, table, [200, 128], ps)) and torch.equal(v[0], _gather(vp, s, table, [200, 128], ps)) and (k != 0).any()
    b16 = [t.view(torch.bfloat16).view(pool // 2, ps, Hkv, d) for t in (kp, vp)]
    table = _i32([[pool // 2 - 1, pool // 2 - 2]])
    k, v, _ = mala.cache_read(*b16, table, _i32([250]), 250)
    assert torch.equal(k[0].view(torch.int16), _gather(b16[0], None, table, [250], ps).view(torch.int16))


def test_reads_of_many_sequences(mala):
    lens = [(x * 7) % 5 for x in range(16384)]
    (kp, vp), _, table = _cache(2, False, lens, 8, 1, 8, extra=0)
    k, v, cu = mala.cache_read(kp, vp, table, _i32(lens), sum(lens))
    pos = torch.cat([torch.arange(n) for n in lens]).cuda()
    seq = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens)).cuda()
    assert torch.equal(k[0], kp[table[seq, pos // 8].long(), pos % 8]) and cu[-1].item() == sum(lens)


# ---- prompts over an e4m3 cache

PROMPTS = [([200, 40, 129], [70, 40, 1]), ([3000], [200]), ([128], [128]), ([50, 0, 300, 10], [0, 0, 300, 10]), ([1], [1]), ([900] * 40, [260] * 40)]


def _keys(kp, vp, ks, vs, table, lens, ps):
    """Keys and values of each request in 64 bits."""
    out = []
    for b, n in enumerate(lens):
        x = torch.arange(n, device="cuda")
        page, at = table[b][x // ps].long(), x % ps
        out.append([t.view(torch.uint8)[page, at].view(torch.float8_e4m3fn).double() * s[page, :, at // 128].double()[..., None] for t, s in ((kp, ks), (vp, vs))])
    return out


@pytest.mark.parametrize("lens,new", PROMPTS)
@pytest.mark.parametrize("ps,Hq,Hkv,d", [(64, 4, 2, 64), (128, 8, 2, 128), (16, 2, 2, 96), (256, 6, 1, 128), (32, 4, 4, 16), (128, 4, 2, 64), (256, 2, 2, 48)])
def test_prompts(mala, lens, new, ps, Hq, Hkv, d):
    """Attention over scale * code in 64 bits: o within the kernels' roundings of P and o to bf16, lse within those of fp32 -- keys and values are not
    rounded on their way."""
    (kp, vp), (ks, vs), table = _cache(11, True, lens, ps, Hkv, d)
    cu = [sum(new[:b]) for b in range(len(new) + 1)]
    q = _randn(4, 1, cu[-1], Hq, d)
    scale, total = 1 / math.sqrt(d), sum(lens)
    o, lse, st = mala.fwd_paged_fp8(q, kp, vp, ks, vs, _i32(cu), table, _i32(lens), max(new), total + 9, scale, 0.0, stats=True)
    assert mala.device_status() == 0 and int(st.totals[0]) == int(st.totals[1])
    for b, (k, v) in enumerate(_keys(kp, vp, ks, vs, table, lens, ps)[:6]):
        for h in range(Hq if new[b] else 0):
            qd = q[0, cu[b]:cu[b + 1], h].double()
            w, z, a = R.attention(qd, k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)], scale)
            parity.check_output(o[0, cu[b]:cu[b + 1], h].double().cpu().numpy(), w.cpu().numpy(), a_ref=a.cpu().numpy())
            # scores: fp32 sums of d products, off by at most (d + 4) 2^-24 of the sum of their magnitudes; exp2 and the sums by a few 2^-23 more
            most = (qd.abs() @ k[:, h // (Hq // Hkv)].abs().T).amax(1) * scale
            err = (lse[h, cu[b]:cu[b + 1]].double() - z).abs()
            assert (err <= (d + 4) * 2.0 ** -24 * most + 2.0 ** -20 * (1 + z.abs())).all(), err.max().item()


def _dequantised(kp, vp, ks, vs, pow2):
    """bf16 pages with the same values (exact where the scales are powers of two)."""
    assert pow2
    out = []
    for t, s in ((kp, ks), (vp, vs)):
        P, ps, Hkv, d = t.shape
        x = t.float().view(P, s.shape[2], -1, Hkv, d) * s.permute(0, 2, 1)[:, :, None, :, None]
        out.append(x.view(P, ps, Hkv, d).to(torch.bfloat16))
    return out


@pytest.mark.parametrize("lens,new", PROMPTS)
@pytest.mark.parametrize("ps,Hq,Hkv,d", [(64, 4, 2, 64), (128, 8, 2, 128), (16, 2, 2, 96), (128, 4, 2, 64)])
@pytest.mark.parametrize("tau", [0.0, 1e-3, 0.05])
def test_prompts_against_bf16_pages(mala, lens, new, ps, Hq, Hkv, d, tau):
    """Scales that are powers of two: the same values lie in bf16 pages, and mala_fwd_paged decides alike, tile by tile."""
    (kp, vp), (ks, vs), table = _cache(11, True, lens, ps, Hkv, d)
    g = torch.Generator(device="cuda").manual_seed(1)
    ks, vs = (2.0 ** -torch.randint(5, 10, t.shape, generator=g, device="cuda").float() for t in (ks, vs))
    cu = [sum(new[:b]) for b in range(len(new) + 1)]
    q = _randn(4, 1, cu[-1], Hq, d) * 2
    most = max(new)
    o, lse, st = mala.fwd_paged_fp8(q, kp, vp, ks, vs, _i32(cu), table, _i32(lens), most, sum(lens), 0.1, tau, stats=True)
    k16, v16 = _dequantised(kp, vp, ks, vs, True)
    o2, lse2, st2 = mala.fwd_paged(q, k16, v16, _i32(cu), table, _i32(lens), most, 0.1, tau, stats=True)
    T = min(st.bitmask.shape[-1], st2.bitmask.shape[-1])
    assert torch.equal(st.bitmask[..., :T], st2.bitmask[..., :T]) and torch.equal(st.totals, st2.totals)
    rows = torch.cat([torch.arange(cu[b], cu[b + 1]) for b in range(len(new))]).cuda()
    a, b, c, e = o[0, rows].double(), o2[0, rows].double(), lse[:, rows], lse2[:, rows]
    assert ((a - b).norm() <= 2.0 ** -8 * 2 * b.norm()) and ((c - e).abs() <= 2.0 ** -20 * (1 + e.abs())).all()


@pytest.mark.parametrize("ps,Hq,Hkv,d,new", [(64, 4, 2, 64, 300), (128, 8, 2, 128, 1500), (16, 2, 2, 96, 40), (128, 4, 2, 64, 300), (256, 4, 2, 64, 2100)])
def test_prompts_that_skip(mala, ps, Hq, Hkv, d, new):
    """Queries that look for their own key: tiles are skipped, the same ones as over bf16 pages of the same values."""
    lens, scale, tau = [2500], 1.0, 1e-3
    (kp, vp), (ks, vs), table = _cache(17, True, lens, ps, Hkv, d)
    ks, vs = torch.full_like(ks, 2.0 ** -7), torch.full_like(vs, 2.0 ** -8)
    k, _, _ = mala.cache_read_fp8(kp, vp, ks, vs, table, _i32(lens), 2500)
    q = k[:, 2500 - new:].repeat_interleave(Hq // Hkv, 2).contiguous()
    args = (_i32([0, new]), table, _i32(lens), new)
    o, lse, st = mala.fwd_paged_fp8(q, kp, vp, ks, vs, *args, 2500, scale, tau, stats=True)
    o2, lse2, st2 = mala.fwd_paged(q, *_dequantised(kp, vp, ks, vs, True), *args, scale, tau, stats=True)
    T = min(st.bitmask.shape[-1], st2.bitmask.shape[-1])
    assert torch.equal(st.bitmask[..., :T], st2.bitmask[..., :T]) and torch.equal(st.totals, st2.totals)
    assert int(st.totals[0]) < int(st.totals[1])      # (tiles are skipped: what the comparison is about)
    assert ((o.double() - o2.double()).norm() <= 2.0 ** -8 * 2 * o2.double().norm()) and ((lse - lse2).abs() <= 2.0 ** -20 * (1 + lse2.abs())).all()


@pytest.mark.parametrize("splits", [2, 5, 33])
@pytest.mark.parametrize("lens,new", PROMPTS)
@pytest.mark.parametrize("ps,Hq,Hkv,d", [(64, 4, 2, 64), (128, 8, 2, 128), (16, 2, 2, 96), (128, 4, 2, 64)])
def test_prompts_in_ranges(mala, lens, new, ps, Hq, Hkv, d, splits):
    """Keys cut into ranges: the tolerances of test_prompts (the merge adds a few roundings in fp32), rows that belong to no sequence
    left as they were, and nothing read that this call did not write."""
    (kp, vp), (ks, vs), table = _cache(11, True, lens, ps, Hkv, d)
    cu = [sum(new[:b]) for b in range(len(new) + 1)]
    q = _randn(4, 1, cu[-1], Hq, d)
    scale, total = 1 / math.sqrt(d), sum(lens)
    ws = torch.full((int(mala.lib().mala_paged_fp8_split_workspace_bytes(len(lens), Hq, Hkv, max(new), total, d, splits)),), 0xff, dtype=torch.uint8, device="cuda")
    o, lse, st = mala.fwd_paged_fp8(q, kp, vp, ks, vs, _i32(cu), table, _i32(lens), max(new), total, scale, 0.0, stats=True, ws=ws, num_splits=splits)
    whole = mala.fwd_paged_fp8(q, kp, vp, ks, vs, _i32(cu), table, _i32(lens), max(new), total, scale, 0.0, stats=True, num_splits=1)[2]
    assert mala.device_status() == 0 and torch.equal(st.totals, whole.totals) and torch.equal(st.bitmask, whole.bitmask) and torch.equal(st.retained, whole.retained)
    for b, (k, v) in enumerate(_keys(kp, vp, ks, vs, table, lens, ps)[:6]):
        for h in range(Hq if new[b] else 0):
            qd = q[0, cu[b]:cu[b + 1], h].double()
            w, z, a = R.attention(qd, k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)], scale)
            parity.check_output(o[0, cu[b]:cu[b + 1], h].double().cpu().numpy(), w.cpu().numpy(), a_ref=a.cpu().numpy())
            most = (qd.abs() @ k[:, h // (Hq // Hkv)].abs().T).amax(1) * scale
            err = (lse[h, cu[b]:cu[b + 1]].double() - z).abs()
            assert (err <= (d + 4) * 2.0 ** -24 * most + 2.0 ** -20 * (1 + z.abs())).all(), err.max().item()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("ps,Hq,Hkv,d,new,splits", [(64, 4, 2, 64, 300, 3), (128, 8, 2, 128, 1500, 4), (16, 2, 2, 96, 40, 7), (128, 4, 2, 64, 300, 3)])
def test_prompts_in_ranges_that_skip(mala, ps, Hq, Hkv, d, new, splits, causal):
    """Every range has a skip test of its own: the tiles that mala_fwd_chunk_split skips over the same values."""
    lens, scale, tau = [2500], 1.0, 1e-3
    (kp, vp), (ks, vs), table = _cache(17, True, lens, ps, Hkv, d)
    ks, vs = torch.full_like(ks, 2.0 ** -7), torch.full_like(vs, 2.0 ** -8)
    k, v, _ = mala.cache_read_fp8(kp, vp, ks, vs, table, _i32(lens), 2500)
    q = k[:, 2500 - new:].repeat_interleave(Hq // Hkv, 2).contiguous()
    o, lse, st = mala.fwd_paged_fp8(q, kp, vp, ks, vs, _i32([0, new]), table, _i32(lens), new, 2500, scale, tau, causal=causal, stats=True, num_splits=splits)
    o2, lse2, st2 = mala.fwd_chunk_split(q, k, v, scale, tau, splits, causal=causal, stats=True)
    T, Q = min(st.bitmask.shape[-1], st2.bitmask.shape[-1]), min(st.bitmask.shape[-2], st2.bitmask.shape[-2])
    assert torch.equal(st.bitmask[..., :Q, :T], st2.bitmask[..., :Q, :T]) and torch.equal(st.totals, st2.totals)
    assert int(st.totals[0]) < int(st.totals[1])
    assert ((o.double() - o2.double()).norm() <= 2.0 ** -8 * 2 * o2.double().norm()) and ((lse - lse2[0]).abs() <= 2.0 ** -20 * (1 + lse2[0].abs())).all()


def test_ranges_leave_rows_and_refuse(mala):
    """Sequences without keys and with more queries than keys keep their rows; counts that the call refuses, and workspaces too small for them."""
    lens, new, ps, Hq, Hkv, d = [0, 500, 30, 257], [5, 40, 31, 257], 64, 4, 2, 64
    (kp, vp), (ks, vs), table = _cache(11, True, lens, ps, Hkv, d)
    cu = _i32([0, 5, 45, 76, 333])
    q = _randn(4, 1, 340, Hq, d)
    L, need = mala.lib(), int(mala.lib().mala_paged_fp8_split_workspace_bytes(4, Hq, Hkv, 257, 787, d, 3))
    o, lse, ws = torch.full_like(q, 7.0), torch.full((Hq, 340), 7.0, device="cuda"), torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")

    def call(splits=3, bytes_=need, B=4):
        return L.mala_fwd_paged_fp8_split(mala._view(q, mala._TIn), mala._view8(kp), mala._view8(vp), ks.data_ptr(), vs.data_ptr(), cu.data_ptr(), table.data_ptr(),
                                          _i32(lens).data_ptr(), mala._view(o, mala._TOut), lse.data_ptr(), None, B, Hq, Hkv, 340, 257, 787, kp.shape[0], ps,
                                          table.shape[1], d, 1, 0.1, 0.0, splits, ws.data_ptr(), bytes_, torch.cuda.current_stream().cuda_stream)
    for kw, code in ((dict(splits=0), -1), (dict(splits=-1), -1), (dict(splits=20000), -2), (dict(bytes_=need - 1), -4), (dict(splits=4), -4)):
        assert call(**kw) == code, kw
    assert (o == 7).all() and (lse == 7).all()
    assert call() == 0 and mala.device_status() == 0
    for a, b in ((0, 5), (45, 76), (333, 340)):
        assert (o[:, a:b] == 7).all() and (lse[:, a:b] == 7).all()
    ref = mala.fwd_paged_fp8(q, kp, vp, ks, vs, cu, table, _i32(lens), 257, 787, 0.1, 0.0, num_splits=1)
    for a, b in ((5, 45), (76, 333)):
        assert ((o[:, a:b].double() - ref[0][:, a:b].double()).norm() <= 2.0 ** -8 * 2 * ref[0][:, a:b].double().norm())
        assert ((lse[:, a:b] - ref[1][:, a:b]).abs() <= 2.0 ** -20 * (1 + ref[1][:, a:b].abs())).all()


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("ps", [64, 128])
@pytest.mark.parametrize("value", [0.0, -0.01, 1e-30, 1e25, 2.0 ** -61, 2.0 ** -60])
def test_prompts_with_far_scales(mala, which, value, ps):
    """Scales that no cache write gives (0, below 0, near the ends of fp32) in some units: bf16(scale * code) there."""
    lens, new, Hq, Hkv, d = [700], [130], 4, 2, 64
    (kp, vp), (ks, vs), table = _cache(13, True, lens, ps, Hkv, d)
    used = table[0, [2, 4 if ps == 128 else 5]].long()
    (ks if which == "k" else vs)[used, 1] = value
    if which == "k" and value > 1:
        for x in used.tolist():            # (finite scores: one key of small codes)
            kp[x] = torch.full_like(kp[x].float(), 2.0 ** -9).to(torch.float8_e4m3fn)
    q = _randn(4, 1, 130, Hq, d)
    o, lse, _ = mala.fwd_paged_fp8(q, kp, vp, ks, vs, _i32([0, 130]), table, _i32(lens), 130, 700, 1 / 8, 0.0)
    k, v, cu = mala.cache_read_fp8(kp, vp, ks, vs, table, _i32(lens), 900)
    o2, lse2, _ = mala.fwd_varlen_prefix(q, k, v, _i32([0, 130]), cu, 130, 700, 1 / 8, 0.0)
    # as finite as the forward over these values.  (Scores of 1e23 are beyond its exponent: fma(s, c, -m) with m = fl(s c) leaves up to |m| 2^-24 = 6e15 instead of
    # 0 for the row's largest score, whatever the cache's type; every other case here is finite in both.)
    assert torch.isfinite(o[torch.isfinite(o2)]).all()
    if value <= 1 or which == "v":
        assert torch.isfinite(o2).all()
    # against keys rounded to bf16 (2^-8 of a key): scores of up to a few units times 2^-8
    if value <= 1 or which == "v":
        assert (lse - lse2).abs().max() <= 0.05 and ((o.double() - o2.double()).norm() <= 0.05 * o2.double().norm())
    assert mala.device_status() == 0


def test_prompts_with_a_workspace_and_refusals(mala):
    lens, ps, Hq, Hkv, d = [90, 200], 64, 4, 2, 64
    (kp, vp), (ks, vs), table = _cache(11, True, lens, ps, Hkv, d)
    q, cu = _randn(4, 1, 60, Hq, d), _i32([0, 20, 60])
    ws = torch.empty(int(mala.lib().mala_paged_fp8_workspace_bytes(2, Hkv, 290, d)), dtype=torch.uint8, device="cuda")
    call = lambda **kw: mala.fwd_paged_fp8(**{**dict(q=q, kpages8=kp, vpages8=vp, kscale=ks, vscale=vs, cu_seqlens_q=cu, block_table=table,  # noqa: E731
                                                     seqlens_k=_i32(lens), max_seqlen_q=40, total_k=290, scale=0.1, tau=0.0), **kw})
    o, lse, _ = call(ws=ws)
    ws.fill_(0xff)                                    # (NaN whichever way it is read)
    assert torch.equal(call(ws=ws)[0], o) and torch.isfinite(o).all()
    assert torch.equal(call(kpages8=kp.view(torch.uint8), vpages8=vp.view(torch.uint8))[0], o)
    for kw in (dict(ws=ws[:-256]), dict(total_k=10), dict(max_seqlen_q=61), dict(scale=0.0), dict(tau=-1.0)):
        with pytest.raises(mala.MalaError):
            call(**kw)
    for kw in (dict(cu_seqlens_q=cu.long()), dict(seqlens_k=_i32([90])), dict(kscale=ks.double()), dict(kscale=ks[:1]), dict(vpages8=vp[:1]), dict(q=q[..., :32]),
               dict(kpages8=kp.float()), dict(q=q.cpu()), dict(block_table=table.cpu())):
        with pytest.raises(AssertionError):
            call(**kw)
    # workspace for fewer keys than there are: the sequences that fit are right, nothing is touched behind the workspace
    total = 150
    part = torch.full((int(mala.lib().mala_paged_fp8_workspace_bytes(2, Hkv, total, d)) + 4096,), 7, dtype=torch.uint8, device="cuda")
    n = part.numel() - 4096
    got = call(total_k=total, ws=part[:n])[0]
    assert torch.equal(got[:, :20], o[:, :20]) and (part[n:] == 7).all() and mala.device_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_a_serving_run_at_rotary_positions(mala, fp8):
    """Requests arrive with prompts, get tokens one by one, finish and make room for others, prompts come behind cached prefixes: tables with
    positions, rotated writes, paged prompts and decode steps, against attention over each request's own rotated keys in 64 bits."""
    ps, Hq, Hkv, d, B, width, pool = 64, 4, 2, 64, 6, 12, 40
    scale = 1 / math.sqrt(d)
    rot = mala.Rotary(mala.rotary_frequencies(48)[0])
    norm = mala.HeadNorm(_randn(1, d) * 0.2 + 1, _randn(2, d) * 0.2 + 1, 1e-5)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    free, count, lens = torch.arange(pool, dtype=torch.int32, device="cuda"), _i32([pool]), _i32([0] * B)
    if fp8:
        kp, vp = (torch.zeros((pool, ps, Hkv, d), dtype=torch.uint8, device="cuda") for _ in range(2))
        ks, vs = (torch.ones((pool, Hkv, 1), device="cuda") for _ in range(2))
    else:
        kp, vp = (torch.zeros((pool, ps, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    keys = [torch.empty((0, Hkv, d), dtype=torch.float64, device="cuda") for _ in range(B)]
    vals = [t.clone() for t in keys]
    for step, new in enumerate([[300, 70, 1, 0, 500, 64], [1] * B, [1] * B, [40, 200, 1, 130, 30, 1], [1] * B]):
        done = [step == 3 and b in (0, 4) for b in range(B)]
        held, c2 = mala.release_pages(torch.tensor(done, device="cuda"), lens, table, free, count, ps)
        rows = sum(new)
        cu, lens, slots, count, pos = mala.page_tables(held, _i32(new), table, free, c2, ps, rows, positions=True)
        x = _randn(100 + step, rows, Hq + 2 * Hkv, d)
        q, k, v = x.split([Hq, Hkv, Hkv], 1)
        if fp8:
            qr = mala.rotary_write_fp8(q, k, v, pos, slots, kp, vp, ks, vs, rot, norm=norm)
        else:
            qr = mala.rotary_write(q, k, v, pos, slots, kp, vp, rot, norm=norm)
        assert (slots >= 0).all()
        kt = R.forward(k, pos, rot.inv_freq, False, 1.0, norm.eps, norm.k_weight)
        at = 0
        for b, n in enumerate(new):
            if done[b]:
                keys[b], vals[b] = keys[b][:0], vals[b][:0]
            keys[b], vals[b] = torch.cat([keys[b], kt[at:at + n]]), torch.cat([vals[b], v[at:at + n].double()])
            at += n
        assert lens.tolist() == [t.shape[0] for t in keys]
        if fp8:
            got = mala.fwd_paged_fp8(qr[None], kp, vp, ks, vs, cu, table, lens, max(new), sum(lens.tolist()), scale, 0.0)[0][0]
            if max(new) == 1:
                dec = mala.decode_fp8_paged(qr[:, None].contiguous(), kp, vp, ks, vs, table, lens, scale, 0.0, 2)[0][:, 0]
        else:
            got = mala.fwd_paged(qr[None], kp, vp, cu, table, lens, max(new), scale, 0.0)[0][0]
            if max(new) == 1:
                dec = mala.decode_paged(qr[:, None].contiguous(), kp, vp, table, lens, scale, 0.0, 2)[0][:, 0]
        at = 0
        for b, n in enumerate(new):
            for h in range(Hq if n else 0):
                want, _, size = R.attention(qr[at:at + n, h].double(), keys[b][:, h // 2], vals[b][:, h // 2], scale)
                for o in (got, dec) if max(new) == 1 else (got,):
                    err = (o[at:at + n, h].double() - want).norm() / want.norm()
                    # bf16: roundings of keys (2^-8 of scores of a few units), P, output; e4m3: keys and values at most 2^-4 each, twice where a scale has grown
                    assert err <= (2 * 2.0 ** -4 if fp8 else 4 * 2.0 ** -8), (step, b, h, err.item())
            at += n
    assert mala.device_status() == 0


def test_a_captured_serving_step(mala):
    """Tables, rotated write and prompts over the e4m3 cache, and the read back, captured once and replayed step by step while the same step runs
    eagerly on another stream: bit for bit the same tables, pages, scales and outputs."""
    ps, Hq, Hkv, d, B, width, pool, rows = 64, 8, 2, 128, 3, 30, 90, 6
    rot = mala.Rotary(mala.rotary_frequencies(128)[0])
    norm = mala.HeadNorm(_randn(1, d) * 0.2 + 1, _randn(2, d) * 0.2 + 1, 1e-5)

    def state():
        return dict(table=torch.full((B, width), -1, dtype=torch.int32, device="cuda"), free=torch.arange(pool, dtype=torch.int32, device="cuda"), count=_i32([pool]),
                    lens=_i32([0] * B), pages=[torch.zeros((pool, ps, Hkv, d), dtype=torch.uint8, device="cuda") for _ in range(2)],
                    scales=[torch.ones((pool, Hkv, 1), device="cuda") for _ in range(2)])

    def step(s, new, x, rows, most, total):
        cu, lens, slots, count, pos = mala.page_tables(s["lens"], new, s["table"], s["free"], s["count"], ps, rows, positions=True)
        q, k, v = x.split([Hq, Hkv, Hkv], 1)
        qr = mala.rotary_write_fp8(q, k, v, pos, slots, *s["pages"], *s["scales"], rot, norm=norm)
        o, lse, _ = mala.fwd_paged_fp8(qr[None], *s["pages"], *s["scales"], cu, s["table"], lens, most, total, 0.1, 0.0)
        read = mala.cache_read_fp8(*s["pages"], *s["scales"], s["table"], lens, total)
        s["lens"].copy_(lens)
        s["count"].copy_(count)
        return qr, o, lse, pos, slots, read[2], read[0][:, :total - 128], read[1][:, :total - 128]
    total = 2200
    first = _randn(5, 2000, Hq + 2 * Hkv, d)
    a, b = state(), state()
    for s in (a, b):
        step(s, _i32([1500, 100, 400]), first, 2000, 1500, 2400)
    for t, u in zip([a["table"], a["lens"], *a["pages"], *a["scales"]], [b["table"], b["lens"], *b["pages"], *b["scales"]]):
        assert torch.equal(t, u)
    x, new = _randn(6, rows, Hq + 2 * Hkv, d), _i32([2, 1, 3])
    side, other, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    held = {n: [t.clone() for t in (v if isinstance(v, list) else [v])] for n, v in a.items()}
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a, new, x, rows, 4, total)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            out = step(a, new, x, rows, 4, total)
    for n, v in a.items():                 # (back to where the other one is)
        for t, u in zip(v if isinstance(v, list) else [v], held[n]):
            t.copy_(u)
    for i, counts in enumerate([[2, 1, 3], [1, 4, 1], [0, 3, 3], [4, 0, 2]]):
        x.copy_(_randn(20 + i, rows, Hq + 2 * Hkv, d))
        new.copy_(_i32(counts))
        mine, mine_new = x.clone(), new.clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            want = step(b, mine_new, mine, rows, 4, total)
        graph.replay()
        torch.cuda.synchronize()
        held_rows = int(a["lens"].sum())
        for j, (t, u) in enumerate(zip(out, want)):
            if j >= 6:                     # (rows behind the last sequence are not written)
                t, u = t[:, :held_rows], u[:, :held_rows]
            assert torch.equal(t, u), (i, j)
        for t, u in zip([a["table"], a["lens"], *a["pages"], *a["scales"]], [b["table"], b["lens"], *b["pages"], *b["scales"]]):
            assert torch.equal(t, u)
    assert mala.device_status() == 0
