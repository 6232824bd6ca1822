"""GPU parity of the calls with a relative position bias at the borders of what they allow: masked keys whose scores lie far above the
visible ones, values that swallow the scores, buckets that begin just above a whole number, gradients far below their neighbours'."""
import math

import numpy as np
import pytest
import torch

from tests import bias_reference as R
from tests import parity
from tests.test_gpu_bias import U, _check, _inputs, _paged, _randn

pytestmark = pytest.mark.gpu
S_ABS = parity.LSE_ABS   # scores in fp32 and their log-sum-exp: the limit of the other calls' tests, for each of the two


@pytest.fixture(scope="module")
def mala():
    from paper_2609_32712_b200 import mala as m
    m.lib()
    return m


def _reference(q, k, v, do, table, scale, nb, md, bidir, causal):
    """One head in 64 bits with the error bounds of its results.  P carries the scores' and the normalizer's error (2 S_ABS, relative)
    and, as an operand, a rounding to bf16; D comes from the bf16 output; every result is rounded once."""
    r = R.head(*(t.double() for t in (q, k, v, table, do)), scale, nb, md, bidir, causal)
    p, _ = R.softmax_rows(r["x"])
    do, k, q, v = (t.double() for t in (do, k, q, v))
    e_o = (U * (r["o"].abs() + r["a"]) * 1.02 + 2 * S_ABS * r["a"]) + 1e-5
    dp = do @ v.T
    off = (dp - (r["o"] * do).sum(-1, keepdim=True)).abs()
    e_ds = p * off * (U + 4 * S_ABS) + p * (e_o * do.abs()).sum(-1, keepdim=True) * 1.02
    sums = lambda t: torch.stack([(t * (r["bk"] == b)).sum() for b in range(nb)])  # noqa: E731
    err = dict(o=e_o, dq=e_ds @ k.abs() * scale, dk=e_ds.T @ q.abs() * scale, dv=(p * (U + 4 * S_ABS)).T @ do.abs(), dtable=sums(e_ds))
    for n in ("dq", "dk", "dv", "dtable"):
        err[n] = err[n] * 1.02 + U * r[n].abs() + 1e-5
    return r, err


@pytest.mark.parametrize("causal,bidir", [(True, False), (False, True)])
@pytest.mark.parametrize("B,H,N,packed", [(1, 2, 300, False), (2, 16, 1300, False), (1, 2, 900, True), (1, 32, 2000, True)])
def test_a_masked_key_far_above_the_others(mala, B, H, N, packed, causal, bidir):
    """Bucket 0 is masked and q = k without a scale: a query's own key, which it does not see, scores about 128 nats, the others 11 or
    so.  One query block per CTA and two, dense and packed."""
    d, nb, md, scale = 128, 32, 128, 1.0
    q, _, v, do, table = _inputs(3 + N + causal, B, H, H, N, N, d, nb)
    k = q.clone()
    table = (table.float() * 0.5).to(torch.bfloat16)
    table[0] = -math.inf
    bias = mala.RelativeBias(table, md, bidir)
    if packed:
        ends = [0, N // 3, N // 3 + 1, N]
        cu = torch.tensor(ends, dtype=torch.int32, device="cuda")
        args = (cu, cu, N - N // 3 - 1, N - N // 3 - 1, bias, scale, 0.0)
        o, lse, _ = mala.fwd_varlen_bias(q, k, v, *args, causal=causal)
        dq, dk, dv, dtable, _ = mala.bwd_varlen_bias(q, k, v, o, do, lse, *args, causal=causal)
        lse = lse[None]
        parts = [(0, slice(a, b)) for a, b in zip(ends, ends[1:])]
    else:
        o, lse, _ = mala.fwd_bias(q, k, v, bias, scale, 0.0, causal=causal)
        dq, dk, dv, dtable, _ = mala.bwd_bias(q, k, v, o, do, lse, bias, scale, 0.0, causal=causal)
        parts = [(b, slice(0, N)) for b in range(B)]
    torch.cuda.synchronize()
    assert mala.device_status() == 0
    for h in sorted({0, H // 2, H - 1}):
        dt = de = 0
        above = 0
        for b, s in parts:
            r, err = _reference(q[b, s, h], k[b, s, h], v[b, s, h], do[b, s, h], table[:, h], scale, nb, md, bidir, causal)
            above += int((q[b, s, h].double().square().sum(-1) - r["x"].max(-1).values > 90).sum())
            _check(o[b, s, h], r["o"], err["o"], f"o {b} {h}")
            empty = torch.isinf(r["lse"])
            assert torch.equal(torch.isinf(lse[b, h, s]), empty)
            assert (lse[b, h, s].double() - r["lse"])[~empty].abs().amax().nan_to_num(0.0).item() <= S_ABS if (~empty).any() else True
            for got, n in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
                _check(got[b, s, h], r[n], err[n], f"{n} {b} {h}")
            dt, de = dt + r["dtable"], de + err["dtable"]
        assert above > 0                                   # (the input is what it is meant to be)
        _check(dtable[:, h], dt, de, f"dtable {h}")


@pytest.mark.parametrize("tau", [0.0, 1e-4])
@pytest.mark.parametrize("Sq,Hq,Hkv,d,page", [(1, 2, 1, 64, 16), (3, 8, 2, 128, 128), (1, 8, 8, 96, 64), (2, 16, 2, 128, 32)])
@pytest.mark.parametrize("case", ["masked near", "masked far", "only far", "lowest near", "lowest far", "lowest everywhere"])
@pytest.mark.parametrize("splits", [1, 3, 14])
def test_decode_with_masked_buckets(mala, case, splits, Sq, Hq, Hkv, d, page, tau):
    """As in a prompt: -inf masks a bucket's keys, also all of a split or of a row; a type's lowest value does too, but a row of nothing
    else weighs its keys alike, however they are divided among the splits."""
    lens, nb, md = [1, 5, 150, 700, 1999], 16, 200
    kp, vp, bt, sl = _paged(7, lens, page, Hkv, d)
    q, table = _randn(8, len(lens), Sq, Hq, d), _randn(9, nb, Hq)
    low = torch.finfo(torch.bfloat16).min
    if case == "masked near":
        table[:5] = -math.inf            # (the first two requests see nothing)
    elif case == "masked far":
        table[nb - 1] = -math.inf        # (the last request's older splits see nothing)
    elif case == "only far":
        table[:nb - 1] = -math.inf
    elif case == "lowest near":
        table[:nb - 1] = low             # (the shortest requests have no other)
    elif case == "lowest far":
        table[nb - 2:] = low
    else:
        table[:] = low
    scale = 1 / math.sqrt(d)
    o, lse, _ = mala.decode_paged_bias(q, kp, vp, bt, sl, mala.RelativeBias(table, md), scale, tau, splits)
    torch.cuda.synchronize()
    assert mala.device_status() == 0
    lse = lse.view(len(lens), Sq, Hq)
    for b, n in enumerate(lens):
        idx = bt[b, :-(-n // page)].long()
        k, v = (t[idx].reshape(-1, Hkv, d)[:n].double() for t in (kp, vp))
        for s in range(Sq):
            seen = n - Sq + s + 1
            for h in range(0, Hq, max(1, Hq // 4)):
                if seen <= 0:
                    assert (o[b, s, h] == 0).all() and lse[b, s, h] == -math.inf
                    continue
                g = h // (Hq // Hkv)
                r = R.head(q[b, s, h:h + 1].double(), k[:seen, g], v[:seen, g], table[:, h].double(), None, scale, nb, md, False, True)
                want = float(r["lse"][0])
                if 1e6 < -want < math.inf:       # (the normalizer's logarithm is below 2^-53 of such a bias: the weights without it)
                    w = torch.softmax(r["x"], -1)
                    r.update(o=w @ v[:seen, g], a=w @ v[:seen, g].abs())
                # (tau: a skipped tile's mass is at most tau of the row's, Proposition 1; a row of lowest values has no tile below another)
                _check(o[b, s, h], r["o"][0], (U + 2 * tau) * (r["o"][0].abs() + r["a"][0]) * 1.02 + 1e-5 + 2 * tau * float(v.abs().max()), f"o {b} {s} {h}")
                if abs(want) < 1e6:
                    assert abs(float(lse[b, s, h]) - want) <= S_ABS + 2 * tau
                else:
                    assert float(lse[b, s, h]) == want if math.isinf(want) else -math.inf < float(lse[b, s, h]) < -1e38


@pytest.mark.parametrize("nb,md,n", [(73, 905, 347), (64, 21228, 9423), (32, 43921, 16325)])
def test_buckets_that_begin_just_above_a_whole_number(mala, nb, md, n):
    """Distance n lies below the start of a bucket by less than 1e-9 of itself.  q = 0 and neighbouring values 8 apart: the output is the
    weight of that one key, which the wrong bucket changes by e^8."""
    starts = R.bucket_starts(nb, md, False)[2]
    assert n + 1 in starts and n not in starts
    table = (torch.arange(nb, device="cuda") % 2 * 8 - 4).to(torch.bfloat16)[:, None].contiguous()
    table[0] = -4
    for at in (n - 1, n, n + 1):
        k = _randn(1, 1, at + 1, 1, 64)
        x, bk = R.scores(torch.zeros((1, 64), dtype=torch.float64, device="cuda"), k[0, :, 0].double(), table[:, 0].double(), 1.0, nb, md, False, True)
        v = torch.zeros_like(k)
        v[0, 0] = 1.0                      # (the key at distance `at`)
        o, _, _ = mala.fwd_bias(torch.zeros_like(k[:, :1]), k, v, mala.RelativeBias(table, md), 1.0, 0.0)
        p, _ = R.softmax_rows(x)
        want = float(p[0, 0])
        assert abs(float(o[0, 0, 0, 0]) / want - 1) <= 3 * U, at     # (two roundings to bf16; the wrong bucket: e^8)


@pytest.mark.parametrize("low", [-1e7, -1e9, -1.7e10, -1e20, -2e38, float(torch.finfo(torch.bfloat16).min)])
@pytest.mark.parametrize("packed", [False, True])
def test_rows_whose_normalizer_has_swallowed_the_scores_get_no_gradient(mala, low, packed):
    """The first rows see nothing but keys whose bias is so low that their lse in fp32 says nothing of the scores any more: no gradient,
    and every other row's as if these were not there."""
    N, d, nb, md, H = 700, 64, 16, 200, 2
    q, k, v, do, table = _inputs(17, 1, H, H, N, N, d, nb)
    table[0:3] = low
    bias = mala.RelativeBias(table, md)
    scale = 1 / math.sqrt(d)
    if packed:
        cu = torch.tensor([0, N], dtype=torch.int32, device="cuda")
        o, lse, _ = mala.fwd_varlen_bias(q, k, v, cu, cu, N, N, bias, scale, 0.0)
        dq, dk, dv, dtable, _ = mala.bwd_varlen_bias(q, k, v, o, do, lse, cu, cu, N, N, bias, scale, 0.0)
    else:
        o, lse, _ = mala.fwd_bias(q, k, v, bias, scale, 0.0)
        dq, dk, dv, dtable, _ = mala.bwd_bias(q, k, v, o, do, lse, bias, scale, 0.0)
    torch.cuda.synchronize()
    assert mala.device_status() == 0
    assert (dq[0, :3] == 0).all()
    rest = do.clone()
    rest[:, :3] = 0
    for h in range(H):
        r, err = _reference(q[0, :, h], k[0, :, h], v[0, :, h], rest[0, :, h], table[:, h], scale, nb, md, False, True)
        for got, n in ((dq[0, :, h], "dq"), (dk[0, :, h], "dk"), (dv[0, :, h], "dv"), (dtable[:, h], "dtable")):
            _check(got, r[n], err[n], f"{n} {h}")


def test_rows_below_that_limit_keep_their_gradient(mala):
    """A bias of -1e4 under all keys of the first rows: lse carries it with half a step of 2^-11, so P does to 2^-10."""
    N, d, nb, md, H = 300, 64, 16, 200, 2
    q, k, v, do, table = _inputs(18, 1, H, H, N, N, d, nb)
    table[:] = -1e4
    bias = mala.RelativeBias(table, md)
    o, lse, _ = mala.fwd_bias(q, k, v, bias, 0.125, 0.0)
    grads = mala.bwd_bias(q, k, v, o, do, lse, bias, 0.125, 0.0)
    for h in range(H):
        r, err = _reference(q[0, :, h], k[0, :, h], v[0, :, h], do[0, :, h], table[:, h], 0.125, nb, md, False, True)
        for got, n in ((grads[0][0, :, h], "dq"), (grads[1][0, :, h], "dk"), (grads[2][0, :, h], "dv"), (grads[3][:, h], "dtable")):
            _check(got, r[n], err[n], f"{n} {h}")


@pytest.mark.parametrize("causal,bidir", [(True, False), (False, True)])
def test_gradient_of_a_bucket_far_below_its_neighbours(mala, causal, bidir):
    """Buckets whose keys weigh 2^-43 of the others': their gradient is a sum of their own terms alone, without what the neighbouring
    diagonals' rounding leaves (2^-24 of far larger sums).  A row's incoming gradient is the value three keys before it, so that all
    terms of bucket 3 have the same sign."""
    N, d, nb, md, H = 600, 64, 32, 128, 2
    q, k, v, do, table = _inputs(61, 1, H, H, N, N, d, nb)
    low = 3
    table[low] -= 30.0
    do = v.roll(low, 1)
    bias = mala.RelativeBias(table, md, bidir)
    o, lse, _ = mala.fwd_bias(q, k, v, bias, 0.125, 0.0, causal=causal)
    dtable = mala.bwd_bias(q, k, v, o, do, lse, bias, 0.125, 0.0, causal=causal)[3]
    for h in range(H):
        r, err = _reference(q[0, :, h], k[0, :, h], v[0, :, h], do[0, :, h], table[:, h], 0.125, nb, md, bidir, causal)
        bound = err["dtable"] - 1e-5               # (nothing absolute: what is left is relative to the bucket's own terms)
        want = float(r["dtable"][low])
        assert 0 < want < 1e-8 and float(bound[low]) < 0.1 * want
        assert abs(float(dtable[low, h]) - want) <= float(bound[low])


@pytest.mark.parametrize("tau", [1e-3, 0.3])
@pytest.mark.parametrize("lq,lk,Hq,Hkv,d,causal", [([333, 0, 1, 517, 900], None, 4, 2, 64, True), ([200, 640, 7], [900, 700, 500], 2, 2, 128, True),
                                                   ([130, 256, 400], [500, 130, 700], 2, 1, 64, False)])
def test_packed_sequences_skip_tiles_like_single_ones(mala, lq, lk, Hq, Hkv, d, causal, tau):
    """Packed, tau > 0: every sequence's masks, output and gradients are those of the call with that sequence alone (whose masks and
    results are compared with the plain implementation elsewhere)."""
    nb, md = 32, 600
    lk = lq if lk is None else lk
    q, k, v, do, table = _inputs(71, 1, Hq, Hkv, sum(lq), sum(lk), d, nb)
    table = (table.float() - torch.arange(nb, device="cuda")[:, None] * 0.5).to(torch.bfloat16)
    cu, ck = (torch.tensor([0] + list(np.cumsum(x)), dtype=torch.int32, device="cuda") for x in (lq, lk))
    scale = 1 / math.sqrt(d)
    bias = mala.RelativeBias(table, md)
    mq, mk = max(lq), max(lk)
    o, lse, fst = mala.fwd_varlen_bias(q, k, v, cu, ck, mq, mk, bias, scale, tau, causal=causal, stats=True)
    dq, dk, dv, dtable, bst = mala.bwd_varlen_bias(q, k, v, o, do, lse, cu, ck, mq, mk, bias, scale, tau, causal=causal, stats=True)
    torch.cuda.synchronize()
    assert mala.device_status() == 0
    Tk = -(-mk // 128)
    fm, bm = fst.mask(Tk).cpu(), bst.mask(-(-(mq + 127) // 128)).cpu()
    sums = torch.zeros((nb, Hq), dtype=torch.float64, device="cuda")
    skipped = 0
    for x, (n, m) in enumerate(zip(lq, lk)):
        if n == 0:
            continue
        a, b = int(cu[x]), int(ck[x])
        qs, ks, vs, ds = q[:, a:a + n], k[:, b:b + m], v[:, b:b + m], do[:, a:a + n]
        o1, lse1, f1 = mala.fwd_bias(qs, ks, vs, bias, scale, tau, causal=causal, stats=True)
        g1 = mala.bwd_bias(qs, ks, vs, o1, ds, lse1, bias, scale, tau, causal=causal, stats=True)
        tq, tk = -(-(n + ((m - n) % 128 if causal else 0)) // 128), -(-m // 128)
        one, back = f1.mask(tk).cpu(), g1[4].mask(tq).cpu()
        assert torch.equal(fm[x, :, :tq, :tk], one[0]) and torch.equal(bm[x, :, :tk, :tq], back[0])
        legal = sum(min(tk, i + 1 + (m - n) // 128) if causal else tk for i in range(tq)) * Hq
        skipped += legal - int(one.sum())
        assert torch.equal(o[:, a:a + n], o1) and torch.equal(lse[:, a:a + n], lse1[0])
        assert torch.equal(dk[:, b:b + m], g1[1]) and torch.equal(dv[:, b:b + m], g1[2])
        # (dQ: fp32 sums in any order, then one rounding, which may go either way)
        assert (dq[:, a:a + n].float() - g1[0].float()).abs().max() <= 2 * U * g1[0].float().abs().max()
        sums += g1[3].double()
    # (the single calls' tables are rounded to bf16 one by one)
    assert ((dtable.double() - sums).abs() <= 2 * U * len(lq) * sums.abs().max()).all()
    # (the bias falls by 15.5 at most, and the largest of a tile's 16384 scores lies about 4 above the others: enough for
    # ln(0.3 / L) = -8, not for ln(1e-3 / L) = -13.7 in sequences that end at 900 keys)
    assert skipped > 0 or tau < 0.1


def test_gradients_of_a_mean_over_the_rows(mala):
    """The incoming gradient of a pooled output is one row for all of them (a stride of 0), and one that starts off 16 bytes is a slice
    of a wider one: the calls take both, with a bias and without."""
    from paper_2609_32712_b200 import autograd as A
    q, k, v, _, table = _inputs(81, 2, 4, 2, 200, 200, 64, 32)
    w = _randn(82, 2, 4, 64)
    wide = _randn(83, 2, 200, 4, 72)
    cu = torch.tensor([0, 60, 200], dtype=torch.int32, device="cuda")
    calls = [(lambda q, k, v, t: A.mala_attention_bias(q, k, v, t, 0.0), 2), (lambda q, k, v, t: A.mala_attention(q, k, v, 0.0), 2),
             (lambda q, k, v, t: A.mala_attention_bias_packed(q, k, v, t, cu, cu, 140, 140, 0.0), 1),
             (lambda q, k, v, t: A.mala_attention_packed(q, k, v, cu, cu, 140, 140, 0.0), 1)]
    for f, B in calls:
        for do in (w[:B, None].expand(B, 200, 4, 64), wide[:B, ..., 1:65]):
            grads = []
            for g in (do, do.contiguous()):
                leaves = [t[:B].clone().requires_grad_(True) for t in (q, k, v)] + [table.clone().requires_grad_(True)]
                f(*leaves).backward(g)
                grads.append([t.grad for t in leaves])
            for x, y in zip(grads[0][1:], grads[1][1:]):
                assert (x is None and y is None) or torch.equal(x, y)
            assert (grads[0][0].float() - grads[1][0].float()).abs().max() <= 2 * U * grads[1][0].float().abs().max()


@pytest.mark.parametrize("case", ["masked near", "masked far", "only far", "lowest near", "lowest far", "lowest everywhere"])
@pytest.mark.parametrize("tau", [1e-3, 0.3])
@pytest.mark.parametrize("N,H,causal", [(700, 2, True), (1500, 30, True), (700, 2, False)])
def test_masked_buckets_with_skipped_tiles(mala, N, H, causal, tau, case):
    """tau > 0: masked and lowest buckets on the tiles that the call says it has retained, one query block per CTA and two."""
    d, nb, md = 64, 16, 200
    q, k, v, do, table = _inputs(19 + N, 1, H, H, N, N, d, nb)
    low = torch.finfo(torch.bfloat16).min
    if case == "masked near":
        table[0:3] = -math.inf
    elif case == "masked far":
        table[nb - 1] = -math.inf
    elif case == "only far":
        table[:nb - 1] = -math.inf
    elif case == "lowest near":
        table[:3] = low
    elif case == "lowest far":
        table[nb - 4:] = low
    else:
        table[:] = low
    bias, scale = mala.RelativeBias(table, md), 1 / math.sqrt(d)
    o, lse, fst = mala.fwd_bias(q, k, v, bias, scale, tau, causal=causal, stats=True)
    dq, dk, dv, dtable, bst = mala.bwd_bias(q, k, v, o, do, lse, bias, scale, tau, causal=causal, stats=True)
    torch.cuda.synchronize()
    assert mala.device_status() == 0
    T = -(-N // 128)
    fm, bm = fst.mask(T).cpu(), bst.mask(T).cpu()
    for h in sorted({0, H - 1}):
        keep = R.expand(torch.where(fm[0, h], 2, 0), N, N).cuda()
        qd, kd, vd, dd, td = (t.double() for t in (q[0, :, h], k[0, :, h], v[0, :, h], do[0, :, h], table[:, h]))
        r = R.head(qd, kd, vd, td, None, scale, nb, md, False, causal, keep)
        x = r["x"]
        # (a row's weights by softmax: beside a lowest value the normalizer's logarithm vanishes in 64 bits too)
        p = torch.where((x == -math.inf).all(1, keepdim=True), torch.zeros_like(x), torch.softmax(x, 1).nan_to_num(0.0))
        ro, ra = p @ vd, p @ vd.abs()
        _check(o[0, :, h], ro, U * (ro.abs() + ra) * 1.02 + 2 * S_ABS * ra + 1e-5, f"o {h}")
        gone = (r["lse"].abs() >= 2.0 ** 20)                 # (nothing visible, or nothing but lowest values: no gradient)
        assert torch.equal(torch.isinf(lse[0, h]), (x == -math.inf).all(1))
        assert (lse[0, h].double() - r["lse"])[~gone].abs().max().item() <= S_ABS if (~gone).any() else True
        # what is skipped weighs no more than Eq. 3 says: a tile's key below tau / L of the normalizer (with the scores' error)
        full, _ = R.scores(qd, kd, td, scale, nb, md, False, causal)
        L = torch.arange(1, N + 1, device="cuda").double() if causal else torch.full((N,), float(N), device="cuda", dtype=torch.float64)
        lost = (~keep) & (full > -math.inf)
        assert ((full - r["lse"][:, None])[lost] <= (torch.log(tau / L)[:, None].expand_as(full))[lost] + 4 * S_ABS).all()
        backkeep = R.expand(torch.where(bm[0, h].T, 2, 0), N, N).cuda()
        xb = torch.where(backkeep, full, torch.full_like(full, -math.inf))
        pb = torch.where(gone[:, None], torch.zeros_like(xb), torch.exp(xb - torch.where(gone, torch.zeros_like(r["lse"]), lse[0, h].double())[:, None]))
        dp = dd @ vd.T
        D = (o[0, :, h].double() * dd).sum(1, keepdim=True)
        ds = pb * (dp - D)
        e_ds = pb * (dp - D).abs() * (U + 4 * S_ABS)
        one = lambda t: torch.stack([(t * (r["bk"] == b)).sum() for b in range(nb)])  # noqa: E731
        for got, want, err, n in ((dq, ds @ kd * scale, e_ds @ kd.abs() * scale, "dq"), (dk, ds.T @ qd * scale, e_ds.T @ qd.abs() * scale, "dk"),
                                  (dv, pb.T @ dd, (pb * (U + 4 * S_ABS)).T @ dd.abs(), "dv")):
            _check(got[0, :, h], want, err * 1.02 + U * want.abs() + 1e-5, f"{n} {h}")
        _check(dtable[:, h], one(ds), one(e_ds) * 1.02 + U * one(ds).abs() + 1e-4, f"dtable {h}")
