"""Prompts over an e4m3 cache at their limits: requests whose cache holds infinities and NaNs beside others, scores whose factors leave fp32, and scales at
the ends of the range that comes in at the softmax and beyond it, against attention in 64 bits."""
import math

import pytest
import torch

from tests import parity
from tests import rotary_reference as R

pytestmark = pytest.mark.gpu

PS, SHAPES = "ps,Hq,Hkv,d", [(64, 4, 2, 64), (128, 4, 2, 64), (128, 8, 2, 128), (16, 32, 8, 96), (128, 32, 8, 64), (256, 32, 4, 128)]   # 32 heads: two blocks of queries per CTA


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


def _cache(seed, lens, ps, Hkv, d):
    per = [-(-n // ps) for n in lens]
    table = torch.full((len(lens), max(per)), -1, dtype=torch.int32)
    order = torch.randperm(sum(per), generator=torch.Generator().manual_seed(seed)).tolist()
    for b, n in enumerate(per):
        table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    pages = [(_randn(seed + x, sum(per), ps, Hkv, d).float() * 100).clamp(-448, 448).to(torch.float8_e4m3fn) for x in range(2)]
    scales = [_randn(seed + 2 + x, sum(per), Hkv, max(1, ps // 128)).float().abs() * 0.01 + 0.005 for x in range(2)]
    return pages, scales, table.cuda()


@pytest.mark.parametrize(PS, SHAPES)
@pytest.mark.parametrize("what", ["value codes", "value scales", "key codes"])
@pytest.mark.parametrize("tau,splits,causal", [(0.0, 1, True), (0.0, 3, True), (0.0, 1, False), (1e-3, 1, True), (1e-3, 2, False)])
def test_requests_do_not_reach_one_another(mala, ps, Hq, Hkv, d, what, tau, splits, causal):
    """NaN codes, and values that are infinite (448 * 1e36), at the front of a request's cache: the requests beside it, whose last blocks are not
    whole, get the results that they have beside a clean one, bit by bit, and the request itself NaNs in the columns that hold them."""
    lens, new, col = [200, 300, 77, 129], [40, 300, 1, 129], 5
    (kp, vp), (ks, vs), table = _cache(3, lens, ps, Hkv, d)
    q, cu = _randn(9, 1, sum(new), Hq, d), [0, 40, 340, 341, 470]

    def call():
        return mala.fwd_paged_fp8(q, kp, vp, ks, vs, _i32(cu), table, _i32(lens), max(new), sum(lens), 1 / math.sqrt(d), tau, causal=causal, num_splits=splits)[:2]
    clean = call()
    if what == "value codes":
        for x in range(0, 300, 7):
            vp.view(torch.uint8)[table[1, x // ps], x % ps, :, col] = 0x7f
    elif what == "value scales":
        vp.view(torch.uint8)[table[1, 0], :, :, col] = 0x7e                  # 448
        vs[table[1, 0].long(), :, 0] = 1e36
    else:
        kp.view(torch.uint8)[table[1, 0], :, :, col] = 0xff
    got = call()
    assert mala.device_status() == 0
    for b in (0, 2, 3):
        rows = slice(cu[b], cu[b + 1])
        assert torch.isfinite(clean[0][:, rows]).all() and torch.equal(got[0][:, rows], clean[0][:, rows]) and torch.equal(got[1][:, rows], clean[1][:, rows]), b
    if tau == 0 and what == "value codes":
        mine = got[0][:, cu[1]:cu[2]]
        assert torch.isnan(mine[..., col]).all() and torch.equal(got[1], clean[1])
        rest = [c for c in range(d) if c != col]
        assert torch.equal(mine[..., rest], clean[0][:, cu[1]:cu[2]][..., rest])


UP = 2.0 ** 60


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("value", [UP, UP * (1 + 2.0 ** -23), 2 * UP, 1e25, 1 / UP, (1 - 2.0 ** -24) / UP, 0.5 / UP])
@pytest.mark.parametrize("ps,splits", [(64, 1), (128, 1), (64, 3), (256, 3)])
def test_scales_at_the_ends(mala, which, value, ps, splits):
    """Scales of 2^-60 and 2^60, which come in at the softmax, and beyond, where values are bf16(scale * code), in some units of a KV head, against
    attention over these values in 64 bits.  Queries are scaled down where keys are large, so that scores stay at a few units."""
    n, new, Hq, Hkv, d = 700, 130, 4, 2, 64
    (kp, vp), (ks, vs), table = _cache(13, [n], ps, Hkv, d)
    (ks if which == "k" else vs)[table[0, [0, 2]].long(), 1] = value
    q = _randn(4, 1, new, Hq, d)
    if which == "k" and value > 1:
        q = (q.float() * 2.0 ** -(round(math.log2(value)) + 7)).to(torch.bfloat16)          # (exact)
    o, lse, _ = mala.fwd_paged_fp8(q, kp, vp, ks, vs, _i32([0, new]), table, _i32([n]), new, n, 1 / 8, 0.0, num_splits=splits)
    x = torch.arange(n, device="cuda")
    page, at = table[0][x // ps].long(), x % ps
    keys = []
    for t, s in ((kp, ks), (vp, vs)):
        code, by = t[page, at].float(), s[page, :, at // 128][..., None]
        apart = (by >= 1 / UP) & (by <= UP)
        keys.append(torch.where(apart, code.double() * by.double(), (code * by).to(torch.bfloat16).double()))
    for h in range(Hq):
        qd, k, v = q[0, :, h].double(), keys[0][:, h // 2], keys[1][:, h // 2]
        w, z, a = R.attention(qd, k, v, 1 / 8)
        assert z.abs().max() < 100                          # (scores of a few units: what the tolerances below are for)
        parity.check_output(o[0, :, h].double().cpu().numpy(), w.cpu().numpy(), a_ref=a.cpu().numpy())
        # as for scales in the middle: fp32 sums of d products, off by at most (d + 4) 2^-24 of the sum of their magnitudes; exp2 and the sums by a few 2^-23 more
        most = (qd.abs() @ k.abs().T).amax(1) / 8
        err = (lse[h].double() - z).abs()
        assert (err <= (d + 4) * 2.0 ** -24 * most + 2.0 ** -20 * (1 + z.abs())).all(), err.max().item()
    assert mala.device_status() == 0


@pytest.mark.parametrize("ps,d", [(64, 64), (128, 64), (128, 128)])
@pytest.mark.parametrize("splits", [1, 2])
def test_scores_whose_factor_is_below_fp32(mala, ps, d, splits):
    """scale * key scale below the least number of fp32: all scores are 0, and masked keys stay masked."""
    n, new, Hq, Hkv = 300, 70, 4, 2
    (kp, vp), (ks, vs), table = _cache(5, [n], ps, Hkv, d)
    ks = torch.full_like(ks, 1 / UP)
    q = _randn(4, 1, new, Hq, d)
    o, lse, _ = mala.fwd_paged_fp8(q, kp, vp, ks, vs, _i32([0, new]), table, _i32([n]), new, n, 1e-30, 0.0, num_splits=splits)
    x = torch.arange(n, device="cuda")
    page, at = table[0][x // ps].long(), x % ps
    v = vp[page, at].double() * vs[page, :, at // 128].double()[..., None]
    for h in range(Hq):
        w, z, a = R.attention(q[0, :, h].double() * 0, v[:, h // 2] * 0, v[:, h // 2], 1.0)
        parity.check_output(o[0, :, h].double().cpu().numpy(), w.cpu().numpy(), a_ref=a.cpu().numpy())
        assert ((lse[h].double() - z).abs() <= 2.0 ** -20 * (1 + z.abs())).all()


@pytest.mark.parametrize("ps,d", [(64, 64), (128, 64), (128, 128)])
def test_scores_of_zero_whose_factor_is_above_fp32(mala, ps, d):
    """scale * key scale above the largest number of fp32, queries of 0: all scores are 0."""
    n, new, Hq, Hkv = 300, 70, 4, 2
    (kp, vp), (ks, vs), table = _cache(5, [n], ps, Hkv, d)
    ks = torch.full_like(ks, UP)
    q = torch.zeros((1, new, Hq, d), dtype=torch.bfloat16, device="cuda")
    o, lse, _ = mala.fwd_paged_fp8(q, kp, vp, ks, vs, _i32([0, new]), table, _i32([n]), new, n, 1e30, 0.0)
    visible = torch.arange(n - new + 1, n + 1, device="cuda").double()
    assert torch.isfinite(o).all() and ((lse.double() - visible.log()).abs() <= 2.0 ** -20 * (1 + visible.log())).all()
