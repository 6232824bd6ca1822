"""GPU parity of attention with a learned relative position bias (mala_fwd_bias, mala_bwd_bias, the packed calls and the
paged decode) against the plain 64-bit implementation in bias_reference.py."""
import math

import numpy as np
import pytest
import torch

from tests import bias_reference as R
from tests import parity

pytestmark = pytest.mark.gpu
U = 2.0 ** -8            # half a step of bf16
# |S| error: d products in fp32, |q.k| <= d * max|q||k| -- with d <= 128 and |q|, |k| <= 5: 128 * 2^-24 * 128 * 25 * scale < 4e-3 at the very
# worst and 1e-5 where signs are random; the limit of the other calls' tests holds here too
LSE_ABS = parity.LSE_ABS


@pytest.fixture(scope="module")
def mala():
    from paper_2609_32712_b200 import mala as m
    m.lib()
    return m


def _randn(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _inputs(seed, B, Hq, Hkv, Nq, Nk, d, nb):
    return (_randn(seed, B, Nq, Hq, d), _randn(seed + 1, B, Nk, Hkv, d), _randn(seed + 2, B, Nk, Hkv, d), _randn(seed + 3, B, Nq, Hq, d),
            _randn(seed + 4, nb, Hq))


def _check(got, want, bound, what):
    got, want, bound = (np.asarray(t.double().cpu()) for t in (got, want, bound))
    assert np.isfinite(got).all(), what
    worst = (np.abs(got - want) - bound).max()
    assert worst <= 0, f"{what}: over its bound by {worst:.3e} (largest error {np.abs(got - want).max():.3e})"


def _check_lse(got, want, what="lse"):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isinf(got), torch.isinf(want)), what
    fine = ~torch.isinf(want)
    if fine.any():
        assert (got - want)[fine].abs().max().item() <= LSE_ABS, what


def _compare(q, k, v, do, table, o, lse, grads, scale, nb, md, bidir, causal, keeps=None):
    """One batch entry or sequence: q [Nq,Hq,d] ..., o, lse [Hq,Nq], grads None or (dq, dk, dv).  Returns the table's
    gradient and its error bound, [nb, Hq] each."""
    Hq, Hkv = q.shape[1], k.shape[1]
    G = Hq // Hkv
    dk, dv = (torch.zeros(k.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    dq = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    dt, de = (torch.zeros((nb, Hq), dtype=torch.float64, device="cuda") for _ in range(2))
    for h in range(Hq):
        keep = None if keeps is None else keeps[h].cuda()
        r = R.head(q[:, h].double(), k[:, h // G].double(), v[:, h // G].double(), table[:, h].double(),
                   None if grads is None else do[:, h].double(), scale, nb, md, bidir, causal, keep)
        _check(o[:, h], r["o"], U * (r["o"].abs() + r["a"]) * 1.02 + 1e-5, f"o head {h}")
        _check_lse(lse[h], r["lse"], f"lse head {h}")
        if grads is not None:
            dq[:, h] = r["dq"]
            dk[:, h // G] += r["dk"]
            dv[:, h // G] += r["dv"]
            dt[:, h], de[:, h] = r["dtable"], r["dtable_err"]
    if grads is not None:
        for got, want, what in zip(grads, (dq, dk, dv), ("dq", "dk", "dv")):
            if k.shape[0] == 1 and what != "dv":     # one key: dS = 0 up to the rounding of the output
                assert got.double().abs().max().item() <= 8 * U * (want.abs().max().item() + float(do.double().abs().max() * v.double().abs().max()) * q.shape[2] * scale)
            else:
                parity.check_grad(got.double().cpu().numpy(), want.cpu().numpy(), what)
    return dt, de


def _check_table(got, dt, de):
    _check(got, dt, (de + U * dt.abs()) * 1.05 + 1e-4, "dtable")


DENSE = [
    # B, Hq, Hkv, Nq, Nk, d, causal, bidir, buckets, max distance
    (1, 2, 1, 1, 1, 64, True, False, 32, 128),
    (2, 2, 2, 1, 300, 64, True, False, 32, 128),
    (1, 4, 2, 333, 333, 64, True, False, 32, 128),
    (1, 4, 2, 333, 333, 64, False, True, 32, 128),
    (1, 2, 1, 512, 512, 128, True, False, 8, 20),
    (2, 2, 2, 200, 777, 128, True, True, 32, 300),
    (1, 2, 2, 777, 200, 64, False, True, 16, 64),
    (1, 2, 2, 300, 129, 128, False, False, 16, 64),
    (1, 4, 1, 1100, 1100, 96, True, False, 128, 4000),
    (1, 2, 2, 900, 900, 40, False, True, 4, 2),
    (1, 1, 1, 1500, 1500, 64, True, False, 2, 65536),
    (4, 16, 4, 1300, 1300, 64, True, False, 32, 128),       # two query blocks per CTA
    (4, 16, 16, 700, 700, 128, False, True, 32, 500),
]


@pytest.mark.parametrize("B,Hq,Hkv,Nq,Nk,d,causal,bidir,nb,md", DENSE)
def test_full_attention(mala, B, Hq, Hkv, Nq, Nk, d, causal, bidir, nb, md):
    q, k, v, do, table = _inputs(7 + Nq + Nk, B, Hq, Hkv, Nq, Nk, d, nb)
    scale = 1 / math.sqrt(d)
    bias = mala.RelativeBias(table, md, bidir)
    o, lse, _ = mala.fwd_bias(q, k, v, bias, scale, 0.0, causal=causal)
    dq, dk, dv, dtable, _ = mala.bwd_bias(q, k, v, o, do, lse, bias, scale, 0.0, causal=causal)
    torch.cuda.synchronize()
    assert mala.device_status() == 0
    dt = de = 0
    for b in range(B):
        t, e = _compare(q[b], k[b], v[b], do[b], table, o[b], lse[b], (dq[b], dk[b], dv[b]), scale, nb, md, bidir, causal)
        dt, de = dt + t, de + e
    _check_table(dtable, dt, de)


def test_without_bias_it_is_the_plain_call(mala):
    """A table of one value shifts the scores of a row alike: the output and the gradients of the call without it."""
    q, k, v, do, table = _inputs(3, 1, 4, 2, 640, 640, 128, 32)
    table.fill_(0.75)
    scale = 1 / math.sqrt(128)
    bias = mala.RelativeBias(table)
    o, lse, _ = mala.fwd_bias(q, k, v, bias, scale, 0.0)
    o2, lse2, _ = mala.fwd(q, k, v, scale, 0.0)
    assert (lse - lse2 - 0.75).abs().max().item() <= 1e-5
    assert (o.float() - o2.float()).abs().max().item() <= 2 * U * o2.float().abs().max().item()


@pytest.mark.parametrize("tau", [1e-3, 0.3])
@pytest.mark.parametrize("Nq,Nk,d,causal,bidir,heads", [(900, 900, 64, True, False, (4, 2)), (500, 1237, 128, True, True, (2, 2)),
                                                        (640, 640, 64, False, True, (2, 1)), (2100, 2100, 64, True, False, (40, 40))])
def test_tiles_are_skipped_on_the_biased_scores(mala, Nq, Nk, d, causal, bidir, heads, tau):
    """Algorithms 1 and 2 with a bias that falls with the distance: masks, results and gradients on the retained tiles."""
    Hq, Hkv = heads
    nb, md = 32, 600
    q, k, v, do, table = _inputs(31, 1, Hq, Hkv, Nq, Nk, d, nb)
    h_ = nb // 2 if bidir else nb
    slope = torch.arange(nb, device="cuda") % h_
    table = (table.float() - slope[:, None] * 0.5).to(torch.bfloat16)
    scale = 1 / math.sqrt(d)
    bias = mala.RelativeBias(table, md, bidir)
    o, lse, fst = mala.fwd_bias(q, k, v, bias, scale, tau, causal=causal, stats=True)
    dq, dk, dv, dtable, bst = mala.bwd_bias(q, k, v, o, do, lse, bias, scale, tau, causal=causal, stats=True)
    torch.cuda.synchronize()
    assert mala.device_status() == 0
    shift = (Nk - Nq) % 128 if causal else 0
    Tq, Tk = -(-(Nq + shift) // 128), -(-Nk // 128)
    fm, bm = fst.mask(Tk).cpu(), bst.mask(Tq).cpu()
    L = torch.arange(Nq, device="cuda").double() + 1 + Nk - Nq if causal else torch.full((Nq,), float(Nk), device="cuda", dtype=torch.float64)
    skipped_f = skipped_b = 0
    G = Hq // Hkv
    for h in range(0, Hq, max(1, Hq // 4)):
        qd, kd, vd, dd, td = q[0, :, h].double(), k[0, :, h // G].double(), v[0, :, h // G].double(), do[0, :, h].double(), table[:, h].double()
        x, _ = R.scores(qd, kd, td, scale, nb, md, bidir, causal)
        mask, crit = R.alg1_mask(x, tau, L, shift=shift)
        got = fm[0, h]
        off = (mask == 2) != got
        assert (mask[off] > 0).all() and (crit[off].abs() <= 2 * parity.MASK_BAND).all()
        skipped_f += int((~got & (mask > 0)).sum())
        keep = R.expand(torch.where(got, 2, 0), Nq, Nk, shift).cuda()
        r = R.head(qd, kd, vd, td, None, scale, nb, md, bidir, causal, keep)
        _check(o[0, :, h], r["o"], U * (r["o"].abs() + r["a"]) * 1.02 + 1e-5, "o")
        _check_lse(lse[0, h], r["lse"])
        # Eq. 4 on the GPU's lse
        c = (x - lse[0, h].double()[:, None]) - torch.log(tau / L)[:, None]
        legal = mask > 0
        back = bm[0, h]
        for i in range(Tq):
            r0, r1 = max(0, i * 128 - shift), min(Nq, (i + 1) * 128 - shift)
            for j in range(Tk):
                if not legal[i, j]:
                    assert not back[j, i]
                    continue
                cc = c[r0:r1, j * 128:(j + 1) * 128].max().item()
                assert bool(back[j, i]) == (cc >= 0) or abs(cc) <= parity.MASK_BAND
                skipped_b += not bool(back[j, i])
        if G == 1:
            keepb = R.expand(torch.where(back.T, 2, 0), Nq, Nk, shift).cuda()
            D = (o[0, :, h].double() * dd).sum(-1)
            g = R.head(qd, kd, vd, td, dd, scale, nb, md, bidir, causal, keepb, lse[0, h].double(), D)
            for t, w, what in ((dq[0, :, h], g["dq"], "dq"), (dk[0, :, h], g["dk"], "dk"), (dv[0, :, h], g["dv"], "dv")):
                parity.check_grad(t.double().cpu().numpy(), w.cpu().numpy(), what)
            _check_table(dtable[:, h], g["dtable"], g["dtable_err"])
    # (with buckets on both sides the bias falls by 7.5 at most, which the largest of a tile's 16384 scores, about 5 above the
    # others, all but makes up for: -2.5 > ln(0.3 / L) = -8)
    assert bidir or (skipped_f > 0 and skipped_b > 0)


@pytest.mark.parametrize("causal,bidir", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("lq,lk,Hq,Hkv,d", [([128, 384, 256], None, 2, 1, 128), ([333, 0, 1, 517, 130], None, 4, 2, 64),
                                            ([5, 200, 0, 64, 7], [133, 200, 90, 500, 7], 2, 2, 64),
                                            ([700] * 30, None, 16, 16, 64)])
def test_packed(mala, lq, lk, Hq, Hkv, d, causal, bidir):
    nb, md = 32, 128
    lk = lq if lk is None else lk
    q, k, v, do, table = _inputs(11, 1, Hq, Hkv, sum(lq), sum(lk), d, nb)
    cu, ck = (torch.tensor([0] + list(np.cumsum(x)), dtype=torch.int32, device="cuda") for x in (lq, lk))
    scale = 1 / math.sqrt(d)
    bias = mala.RelativeBias(table, md, bidir)
    o, lse, _ = mala.fwd_varlen_bias(q, k, v, cu, ck, max(lq), max(lk), bias, scale, 0.0, causal=causal)
    dq, dk, dv, dtable, _ = mala.bwd_varlen_bias(q, k, v, o, do, lse, cu, ck, max(lq), max(lk), bias, scale, 0.0, causal=causal)
    torch.cuda.synchronize()
    assert mala.device_status() == 0
    dt = de = torch.zeros((nb, Hq), dtype=torch.float64, device="cuda")
    for x, (n, m) in enumerate(zip(lq, lk)):
        a, b = int(cu[x]), int(ck[x])
        if n == 0:
            assert (dk[0, b:b + m] == 0).all() and (dv[0, b:b + m] == 0).all()
            continue
        if x > 4 and x % 7:
            t, e = _compare_table_only(q[0, a:a + n], k[0, b:b + m], v[0, b:b + m], do[0, a:a + n], table, scale, nb, md, bidir, causal)
        else:
            t, e = _compare(q[0, a:a + n], k[0, b:b + m], v[0, b:b + m], do[0, a:a + n], table, o[0, a:a + n], lse[:, a:a + n],
                            (dq[0, a:a + n], dk[0, b:b + m], dv[0, b:b + m]), scale, nb, md, bidir, causal)
        dt, de = dt + t, de + e
    _check_table(dtable, dt, de)


def _compare_table_only(q, k, v, do, table, scale, nb, md, bidir, causal):
    G = q.shape[1] // k.shape[1]
    r = [R.head(q[:, h].double(), k[:, h // G].double(), v[:, h // G].double(), table[:, h].double(), do[:, h].double(), scale, nb, md, bidir, causal)
         for h in range(q.shape[1])]
    return torch.stack([x["dtable"] for x in r], 1), torch.stack([x["dtable_err"] for x in r], 1)


@pytest.mark.parametrize("causal", [True, False])
def test_sequences_without_keys_get_zeros(mala, causal):
    lq, lk = [40, 300, 130], [40, 0, 130]
    q, k, v, do, table = _inputs(5, 1, 2, 2, sum(lq), sum(lk), 64, 32)
    cu, ck = (torch.tensor([0] + list(np.cumsum(x)), dtype=torch.int32, device="cuda") for x in (lq, lk))
    bias = mala.RelativeBias(table)
    if causal:                      # (the longest sequence has to have as many keys as queries)
        mq, mk = 300, 300
        k, v = (torch.cat([t, t], 1) for t in (k, v))
        k, v = (torch.cat([t, t], 1)[:, :340] for t in (k, v))
    else:
        mq, mk = 300, 130
    o, lse, _ = mala.fwd_varlen_bias(q, k, v, cu, ck, mq, mk, bias, 0.125, 0.0, causal=causal)
    dq, _, _, dtable, _ = mala.bwd_varlen_bias(q, k, v, o, do, lse, cu, ck, mq, mk, bias, 0.125, 0.0, causal=causal)
    torch.cuda.synchronize()
    assert (o[0, 40:340] == 0).all() and (lse[:, 40:340] == -math.inf).all() and (dq[0, 40:340] == 0).all()
    assert torch.isfinite(o.float()).all() and torch.isfinite(dtable.float()).all()
    t = e = 0
    for a, b, n in ((0, 0, 40), (340, 40, 130)):
        x, y = _compare(q[0, a:a + n], k[0, b:b + n], v[0, b:b + n], do[0, a:a + n], table, o[0, a:a + n], lse[:, a:a + n], None, 0.125, 32, 128, False, causal)
        x, y = _compare_table_only(q[0, a:a + n], k[0, b:b + n], v[0, b:b + n], do[0, a:a + n], table, 0.125, 32, 128, False, causal)
        t, e = t + x, e + y
    _check_table(dtable, t, e)


@pytest.mark.parametrize("case", ["masked near", "masked far", "lowest far", "only far", "lowest everywhere", "nan behind the mask"])
def test_masked_buckets(mala, case):
    """-inf masks the keys of a bucket, also all that a row sees; a type's lowest value does too, but a row of nothing else
    weighs them alike; a NaN that no visible key has stays out."""
    N, d, nb, md = 700, 64, 16, 200
    q, k, v, do, table = _inputs(17, 1, 2, 2, N, N, d, nb)
    bidir = case == "nan behind the mask"
    low = torch.finfo(torch.bfloat16).min
    if case == "masked near":
        table[0:3] = -math.inf         # the first rows see nothing
    elif case == "masked far":
        table[nb - 1] = -math.inf
    elif case == "lowest far":
        table[nb - 4:] = low
    elif case == "only far":
        table[:nb - 1] = -math.inf
    elif case == "lowest everywhere":
        table[:] = low
    else:
        table[nb // 2:] = math.nan     # the buckets of later keys, in a causal call
    bias = mala.RelativeBias(table, md, bidir)
    scale = 1 / math.sqrt(d)
    o, lse, _ = mala.fwd_bias(q, k, v, bias, scale, 0.0)
    dq, dk, dv, dtable, _ = mala.bwd_bias(q, k, v, o, do, lse, bias, scale, 0.0)
    torch.cuda.synchronize()
    for t in (o, dq, dk, dv, dtable):
        assert torch.isfinite(t.float()).all()
    ref = torch.where(torch.isnan(table), torch.zeros_like(table), table)
    if case == "lowest everywhere":    # the scores vanish beside it: the mean of the visible values
        want = v[0].double().cumsum(0) / torch.arange(1, N + 1, device="cuda")[:, None, None]
        a = v[0].double().abs().cumsum(0) / torch.arange(1, N + 1, device="cuda")[:, None, None]
        _check(o[0], want, U * (want.abs() + a) * 1.02 + 1e-5, "o")
        return
    dt, de = _compare(q[0], k[0], v[0], do[0], ref, o[0], lse[0], (dq[0], dk[0], dv[0]), scale, nb, md, bidir, True)
    _check_table(dtable, dt, de)
    if case == "masked near":
        assert (o[0, :3] == 0).all() and (lse[0, :, :3] == -math.inf).all() and (dq[0, :3] == 0).all()


def test_borders_of_the_buckets(mala):
    """q = 0: a row's lse is that of its buckets' values alone, so that a distance in the wrong bucket shows."""
    for nb, md, bidir in ((32, 128, False), (32, 128, True), (10, 1000, False), (7, 50, False), (128, 65536, False), (24, 768, True)):
        N = 1100
        q = torch.zeros((1, N, 1, 64), dtype=torch.bfloat16, device="cuda")
        k = _randn(1, 1, N, 1, 64)
        table = (torch.arange(nb, device="cuda") % 2 * 8 - 4).to(torch.bfloat16)[:, None].contiguous()   # neighbours differ by 8
        _, lse, _ = mala.fwd_bias(q, k, k, mala.RelativeBias(table, md, bidir), 1.0, 0.0, causal=False)
        x, _ = R.scores(q[0, :, 0].double(), k[0, :, 0].double(), table[:, 0].double(), 1.0, nb, md, bidir, False)
        # one key in the wrong bucket changes a sum of at most N e^4 by e^4 - e^-4: over 9e-4 of it; fp32 sums of N terms are within 1e-5
        assert (lse[0, 0].double() - torch.logsumexp(x, 1)).abs().max().item() <= 3e-4, (nb, md, bidir)


def test_strides_and_columns(mala):
    """q, k, v as views of one projection, a table that is a slice of a larger one."""
    N, H, d = 400, 4, 64
    x = _randn(23, 1, N, 3 * H, d)
    q, k, v = x[:, :, :H], x[:, :, H:2 * H], x[:, :, 2 * H:]
    big = _randn(24, 40, 9)
    table = big[3:35, 5:9]
    bias = mala.RelativeBias(table, 128, True)
    o, lse, _ = mala.fwd_bias(q, k, v, bias, 0.125, 0.0, causal=False)
    o2, lse2, _ = mala.fwd_bias(q.contiguous(), k.contiguous(), v.contiguous(), mala.RelativeBias(table.contiguous(), 128, True), 0.125, 0.0, causal=False)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    _compare(q[0], k[0], v[0], None, table, o[0], lse[0], None, 0.125, 32, 128, True, False)


def test_table_gradient_is_reproducible(mala):
    q, k, v, do, table = _inputs(41, 2, 8, 2, 1000, 1000, 64, 32)
    bias = mala.RelativeBias(table)
    o, lse, _ = mala.fwd_bias(q, k, v, bias, 0.125, 0.0)
    a = [mala.bwd_bias(q, k, v, o, do, lse, bias, 0.125, 0.0)[1:4] for _ in range(3)]
    for x in a[1:]:
        assert all(torch.equal(s, t) for s, t in zip(a[0], x))


def test_captured_on_a_side_stream(mala):
    """Forward and backward captured once and replayed on new contents of the same buffers, the table's among them."""
    q, k, v, do, table = _inputs(51, 1, 4, 2, 500, 500, 64, 32)
    bias = mala.RelativeBias(table)
    args = (0.125, 0.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o, lse, _ = mala.fwd_bias(q, k, v, bias, *args)
        mala.bwd_bias(q, k, v, o, do, lse, bias, *args)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            o, lse, _ = mala.fwd_bias(q, k, v, bias, *args)
            out = (o, lse) + mala.bwd_bias(q, k, v, o, do, lse, bias, *args)[:4]
    torch.cuda.current_stream().wait_stream(s)
    for seed in (61, 71):
        for t, x in zip((q, k, v, do, table), _inputs(seed, 1, 4, 2, 500, 500, 64, 32)):
            t.copy_(x)
        g.replay()
        torch.cuda.synchronize()
        o2, lse2, _ = mala.fwd_bias(q, k, v, bias, *args)
        want = (o2, lse2) + mala.bwd_bias(q, k, v, o2, do, lse2, bias, *args)[:4]
        for x, y in zip(out[:2] + out[3:], want[:2] + want[3:]):
            assert torch.equal(x, y)
        assert (out[2].float() - want[2].float()).abs().max() <= 2 * U * want[2].float().abs().max()   # (dQ: reductions in any order)


def test_two_streams_at_once(mala):
    """The same calls with different tables and inputs on two streams, many in flight on each: what each returns alone."""
    sets = [_inputs(81, 1, 4, 2, 700, 700, 64, 32), _inputs(91, 2, 4, 4, 260, 900, 128, 16)]
    args = [(0.125, 0.0), (0.09, 1e-4)]

    def run(i):
        q, k, v, do, table = sets[i]
        bias = mala.RelativeBias(table, bidirectional=bool(i))
        o, lse, _ = mala.fwd_bias(q, k, v, bias, *args[i])
        return (o, lse) + mala.bwd_bias(q, k, v, o, do, lse, bias, *args[i])[1:4]
    want = [run(0), run(1)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(10):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i].append(run(i))
    torch.cuda.synchronize()
    for i in (0, 1):
        for one in got[i]:
            assert all(torch.equal(x, y) for x, y in zip(one, want[i]))


def test_a_second_derivative_is_refused(mala):
    from paper_2609_32712_b200.autograd import mala_attention_bias
    q, k, v, _, table = (t.requires_grad_() for t in _inputs(97, 1, 2, 2, 20, 20, 64, 32))
    (dq,) = torch.autograd.grad(mala_attention_bias(q, k, v, table, 0.0).float().square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        dq.float().sum().backward()


def test_tensors_elsewhere_are_refused(mala):
    q, k, v, do, table = _inputs(95, 1, 2, 2, 20, 20, 64, 32)
    for x, y in ((q, k.cpu()), (q.cpu(), k)):
        with pytest.raises(AssertionError):
            mala.fwd_bias(x, y, v, mala.RelativeBias(table), 0.125, 0.0)
    with pytest.raises(AssertionError):
        mala.fwd_bias(q, k, v, mala.RelativeBias(table.cpu()), 0.125, 0.0)
    with pytest.raises(AssertionError):
        mala.cache_write(k[0], v[0], torch.arange(20), k.view(1, 20, 2, 64)[:, :16], v[:, :16])


def _paged(seed, lens, page, Hkv, d):
    per = [-(-n // page) for n in lens]
    pool = sum(per) + 3
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(per + [1]) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    return _randn(seed + 1, pool, page, Hkv, d), _randn(seed + 2, pool, page, Hkv, d), table, torch.tensor(lens, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("tau", [0.0, 1e-4])
@pytest.mark.parametrize("lens,Hq,Hkv,d,page,Sq,bidir,nb,md,splits", [
    ([1], 2, 1, 64, 16, 1, False, 32, 128, 1),
    ([1000, 0, 1, 129, 4097], 8, 2, 128, 128, 1, False, 32, 128, 3),
    ([700, 3, 0, 128], 8, 2, 128, 16, 4, False, 32, 128, 2),
    ([700, 300, 5], 4, 4, 64, 64, 2, True, 32, 600, 4),
    ([2500, 2000], 16, 1, 96, 256, 1, False, 64, 3000, 5),
    ([2500, 77], 1, 1, 128, 32, 1, False, 4, 3, 2),
])
def test_decode_paged(mala, lens, Hq, Hkv, d, page, Sq, bidir, nb, md, splits, tau):
    kp, vp, bt, sl = _paged(77, lens, page, Hkv, d)
    B = len(lens)
    q, table = _randn(78, B, Sq, Hq, d), _randn(79, nb, Hq)
    scale = 1 / math.sqrt(d)
    o, lse, _ = mala.decode_paged_bias(q, kp, vp, bt, sl, mala.RelativeBias(table, md, bidir), scale, tau, splits)
    torch.cuda.synchronize()
    assert mala.device_status() == 0
    lse = lse.view(B, Sq, Hq)
    for b, n in enumerate(lens):
        idx = bt[b, :-(-n // page)].long()
        k, v = (t[idx].reshape(-1, Hkv, d)[:n].double() for t in (kp, vp))
        for s in range(Sq):
            seen = n - Sq + s + 1
            if seen <= 0:
                assert (o[b, s] == 0).all() and (lse[b, s] == -math.inf).all()
                continue
            for h in range(Hq):
                g = h // (Hq // Hkv)
                r = R.head(q[b, s, h:h + 1].double(), k[:seen, g], v[:seen, g], table[:, h].double(), None, scale, nb, md, bidir, True)
                # (tau: a skipped tile's mass is at most tau of the row's, Proposition 1: its values count for tau (|o| + a))
                extra = 0.0 if tau == 0 else tau * 2
                _check(o[b, s, h], r["o"][0], (U + extra) * (r["o"][0].abs() + r["a"][0]) * 1.02 + 1e-5 + extra * float(v.abs().max()), f"o {b} {s} {h}")
                assert abs(float(lse[b, s, h]) - float(r["lse"][0])) <= LSE_ABS + 2 * tau


def test_autograd_functions(mala):
    """The differentiable calls give the kernels' gradients to q, k, v and the table, dense and packed."""
    from paper_2609_32712_b200.autograd import mala_attention_bias, mala_attention_bias_packed
    q, k, v, do, table = _inputs(91, 2, 4, 2, 300, 300, 64, 32)
    leaves = [t.requires_grad_(True) for t in (q, k, v, table)]
    o = mala_attention_bias(q, k, v, table, 0.0, max_distance=100, bidirectional=True, causal=False)
    o.backward(do)
    bias = mala.RelativeBias(table.detach(), 100, True)
    o2, lse, _ = mala.fwd_bias(q.detach(), k.detach(), v.detach(), bias, 0.125, 0.0, causal=False)
    want = mala.bwd_bias(q.detach(), k.detach(), v.detach(), o2, do, lse, bias, 0.125, 0.0, causal=False)
    assert torch.equal(o.detach(), o2)
    for t, w in zip(leaves[1:], want[1:4]):
        assert torch.equal(t.grad, w)
    assert (q.grad.float() - want[0].float()).abs().max() <= 2 * U * want[0].float().abs().max()
    cu = torch.tensor([0, 100, 300], dtype=torch.int32, device="cuda")
    x = [t.detach()[:1].clone().requires_grad_(True) for t in (q, k, v)] + [table.detach().clone().requires_grad_(True)]
    o = mala_attention_bias_packed(*x, cu, cu, 200, 200, 0.0, max_distance=100)
    # (a gradient whose last dimension is not contiguous)
    o.backward(do[:1].transpose(2, 3).contiguous().transpose(2, 3))
    bias = mala.RelativeBias(x[3].detach(), 100)
    y = [t.detach() for t in x[:3]]
    o2, lse, _ = mala.fwd_varlen_bias(*y, cu, cu, 200, 200, bias, 0.125, 0.0)
    want = mala.bwd_varlen_bias(*y, o2, do[:1].contiguous(), lse, cu, cu, 200, 200, bias, 0.125, 0.0)
    assert torch.equal(o.detach(), o2)
    for t, w in zip(x[1:], want[1:4]):
        assert torch.equal(t.grad, w)


def test_table_gradient_by_differences(mala):
    """The gradient of sum(o * do) with respect to a bucket's entry against the difference of two forwards, whose outputs carry
    half a step of bf16 each: sum |do| u (|o| + a) of both over twice the step, plus the table's own rounding."""
    B, H, N, d, nb, md = 1, 2, 500, 64, 16, 60
    q, k, v, do, table = _inputs(95, B, H, H, N, N, d, nb)
    table = torch.round(table.float() * 4).div(4).to(torch.bfloat16)       # (so that the steps are exact)
    bias = mala.RelativeBias(table, md)
    o, lse, _ = mala.fwd_bias(q, k, v, bias, 0.125, 0.0)
    dtable = mala.bwd_bias(q, k, v, o, do, lse, bias, 0.125, 0.0)[3].double()
    step = 0.25
    for b in (0, 3, 8, nb - 1):
        two = []
        for sgn in (1, -1):
            t = table.clone()
            t[b] += sgn * step
            x = mala.fwd_bias(q, k, v, mala.RelativeBias(t, md), 0.125, 0.0)[0].double()
            two.append((x * do.double()).sum((0, 1, 3)))
        for h in range(H):
            # the same difference in 64 bits: how far a step of that size is from the derivative, and the outputs' error bound
            err, exact = 0.0, []
            for sgn in (1, -1):
                t = table[:, h].double().clone()
                t[b] += sgn * step
                r = R.head(q[0, :, h].double(), k[0, :, h].double(), v[0, :, h].double(), t, None, 0.125, nb, md, False, True)
                exact.append((r["o"] * do[0, :, h].double()).sum())
                # (independent roundings: the root of the sum of squares, six times)
                err += 6 * float(((U * (r["o"].abs() + r["a"]) * do[0, :, h].double().abs()) ** 2).sum().sqrt())
            got, want = (two[0][h] - two[1][h]) / (2 * step), (exact[0] - exact[1]) / (2 * step)
            assert abs(float(got - want)) <= err / (2 * step)
            r = R.head(q[0, :, h].double(), k[0, :, h].double(), v[0, :, h].double(), table[:, h].double(), do[0, :, h].double(), 0.125, nb, md, False, True)
            curvature = abs(float(want - r["dtable"][b]))
            assert abs(float(got - dtable[b, h])) <= err / (2 * step) + curvature + float(r["dtable_err"][b]) * 1.05 + U * abs(float(dtable[b, h])) + 1e-4


@pytest.mark.parametrize("top", [3.0, 40.0, 90.0, 3e4, 1e10])
def test_values_far_apart(mala, top):
    """Heads whose values are so far apart that they go by sums, beside heads that go by factors."""
    B, H, N, d, nb, md = 1, 4, 600, 64, 32, 128
    q, k, v, do, table = _inputs(101, B, H, H, N, N, d, nb)
    table[5:9, 0] -= top
    table[nb - 1, 1] += top
    table[2, 2] = -top
    for causal, bidir in ((True, False), (False, True)):
        bias = mala.RelativeBias(table, md, bidir)
        o, lse, _ = mala.fwd_bias(q, k, v, bias, 0.125, 0.0, causal=causal)
        dq, dk, dv, dtable, _ = mala.bwd_bias(q, k, v, o, do, lse, bias, 0.125, 0.0, causal=causal)
        for t in (o, dq, dk, dv, dtable):
            assert torch.isfinite(t.float()).all()
        for h in range(H):
            if top > 1e3 and h == 1:
                continue        # (x = s + top in fp32 keeps no digits of s: compared below 2^10 alone)
            r = R.head(q[0, :, h].double(), k[0, :, h].double(), v[0, :, h].double(), table[:, h].double(), do[0, :, h].double(), 0.125, nb, md, bidir, causal)
            _check(o[0, :, h], r["o"], U * (r["o"].abs() + r["a"]) * 1.02 + 1e-5, f"o head {h}")
            assert (lse[0, h].double() - r["lse"]).abs().max() <= LSE_ABS
            _check_table(dtable[:, h], r["dtable"], r["dtable_err"])
            for got, want in ((dq, r["dq"]), (dk, r["dk"]), (dv, r["dv"])):
                parity.check_grad(got[0, :, h].double().cpu().numpy(), want.cpu().numpy(), f"head {h}")
