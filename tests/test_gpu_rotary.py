"""Rotary positions on the GPU against the formulas in 64 bits: forward and backward, norms, layouts, packed sequences, and the form of a
serving step, into bf16 and e4m3 pages.

Tolerances.  An output is rounded once to bf16: half a step, 2^-8 of its value.  Before that: fp32 products of angles good to 2^-31 turns whose
cos and sin are good to 2^-23 (rounding, and the series' rest of 2.5e-8), a norm whose sum of up to 256 squares has at most 8 + 5 roundings
one behind the other, and the products with it: together below 2^-19 of the magnitudes that the two terms of an output have (of the
three terms of a gradient: R.backward_size)."""
import math

import pytest
import torch

from tests import rotary_reference as R

pytestmark = pytest.mark.gpu

HALF, FP32 = 2.0 ** -8, 2.0 ** -19


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


def _close(got, want, size, half=HALF):
    err = (got.double() - want).abs()
    assert torch.isfinite(err).all()
    bad = err > half * want.abs() + FP32 * size
    assert not bad.any(), (err[bad].max().item(), want[bad][0].item(), int(bad.sum()))


def _check_dw(got, terms, want, total, chain):
    """A weight's gradient: fp32 sums of terms each good to 2^-19, `chain` additions one behind the other."""
    err = (got.double() - want).abs()
    assert (err <= total * (FP32 + chain * 2.0 ** -24) + 1e-30).all(), (err / total).max().item()


def _rule(mala, R_, base=10000.0, interleaved=False, magnitude=1.0):
    f = base ** (-2 * torch.arange(R_ // 2, dtype=torch.float64, device="cuda") / R_)
    return mala.Rotary(f, interleaved=interleaved, magnitude=magnitude)


def _norm(mala, d, seed, fp32=False, eps=1e-5):
    w = [(_randn(seed + x, d).float() * 0.3 + 1).to(torch.float32 if fp32 else torch.bfloat16) for x in (0, 1)]
    return mala.HeadNorm(*w, eps)


def _args(rot, norm, which, pos):
    w = None if norm is None else (norm.q_weight, norm.k_weight)[which]
    return (pos, rot.inv_freq, rot.interleaved, rot.magnitude, None if norm is None else norm.eps, w)


# (head size, rotated columns): all of the head, parts, halves that begin inside a lane's eight columns, single pairs
SIZES = [(128, 128), (128, 64), (128, 32), (64, 64), (64, 16), (80, 20), (80, 40), (80, 80), (96, 24), (96, 96), (256, 256), (256, 64), (8, 8), (8, 2), (16, 6),
         (248, 246), (72, 2), (128, 16), (40, 22)]


@pytest.mark.parametrize("d,rotary", SIZES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("normed", [False, True])
def test_forward_and_backward(mala, d, rotary, interleaved, normed):
    B, Nq, Nk, Hq, Hkv = 2, 5, 9, 6, 3
    rot = _rule(mala, rotary, interleaved=interleaved, magnitude=1.25 if d % 3 else 1.0)
    norm = _norm(mala, d, 7, fp32=d % 16 == 0) if normed else None
    x = _randn(d + rotary, B, Nk, Hq + 2 * Hkv, d)                 # one projection's output: strided parts
    q, k = x[:, Nk - Nq:, :Hq], x[:, :, Hq:Hq + Hkv]
    pos = torch.arange(Nk, device="cuda").expand(B, -1)
    qo, ko = mala.rotary(q, k, rot, norm=norm)
    dq, dk = _randn(1, B, Nq, Hq, d), _randn(2, B, Nk, Hkv, d)
    got = mala.rotary_bwd(dq, dk, rot, norm=norm, q=q, k=k)
    for which, (t, to, g, gx, gw, p) in enumerate(((q, qo, dq, got[0], got[2], pos[:, Nk - Nq:]), (k, ko, dk, got[1], got[3], pos))):
        a = _args(rot, norm, which, p)
        _close(to, R.forward(t, *a), R.size(t, *a))
        want, dw, total = R.backward(g, t, *a)
        _close(gx, want, R.backward_size(g, t, *a))
        assert (gw is None) == (norm is None)
        if norm is not None:
            _check_dw(gw, None, dw, total, t.shape[2] + 32)
    assert mala.device_status() == 0


@pytest.mark.parametrize("B,N,Hq,Hkv,d", [(1, 1, 1, 1, 128), (1, 1, 32, 8, 128), (3, 700, 5, 1, 64), (1, 6001, 33, 8, 128), (70000, 1, 2, 1, 16), (1, 9, 300, 17, 256),
                                          (2, 20000, 3, 2, 32), (1, 12000, 16, 4, 256)])    # (the last one: more than a round of blocks)
@pytest.mark.parametrize("normed", [False, True])
def test_sizes(mala, B, N, Hq, Hkv, d, normed):
    rot, norm = _rule(mala, d), _norm(mala, d, 3) if normed else None
    q, k, dq, dk = (_randn(x, B, N, h, d) for x, h in ((1, Hq), (2, Hkv), (3, Hq), (4, Hkv)))
    pos = torch.arange(N, device="cuda").expand(B, -1)
    qo, ko = mala.rotary(q, k, rot, norm=norm)
    got = mala.rotary_bwd(dq, dk, rot, norm=norm, q=q, k=k)
    rows = max(1, N * B // (8 * 4 * 100))                          # at least: rows that a warp of 4 x 100 blocks takes
    for which, (t, to, g, gx, gw) in enumerate(((q, qo, dq, got[0], got[2]), (k, ko, dk, got[1], got[3]))):
        a = _args(rot, norm, which, pos)
        _close(to, R.forward(t, *a), R.size(t, *a))
        want, dw, total = R.backward(g, t, *a)
        _close(gx, want, R.backward_size(g, t, *a))
        if normed:
            _check_dw(gw, None, dw, total, t.shape[2] * (rows + 1) + 32)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(mala, interleaved):
    """Any int32 position, to the accuracy of near ones (angles of up to 2^31 radians)."""
    pos = torch.tensor([[0, 1, -1, 131071, 1000003, 2 ** 24 + 1, 2 ** 30 + 7, 2 ** 31 - 1, -2 ** 31, -12345678]], device="cuda")
    rot = _rule(mala, 64, interleaved=interleaved)
    q, k = _randn(5, 1, 10, 2, 64), _randn(6, 1, 10, 2, 64)
    qo, ko = mala.rotary(q, k, rot, positions=pos.to(torch.int32))
    # angles from whole numbers: f in units of 2^-80, the product modulo a turn without any rounding
    tau = 2 * math.pi
    exact = torch.empty((1, 10, 32), dtype=torch.float64)
    from fractions import Fraction
    pi = Fraction(314159265358979323846264338327950288419716939937510582097494459230781640628620899, 10 ** 80)
    for r, n in enumerate(pos[0].tolist()):
        for i, f in enumerate(rot.inv_freq.tolist()):
            turns = Fraction(f) * n / (2 * pi)
            exact[0, r, i] = float(turns - round(turns)) * tau
    exact = exact.cuda()
    for t, got in ((q, qo), (k, ko)):
        y1, y2 = R.split(t.double(), 64, interleaved)
        c, s = exact.cos()[:, :, None], exact.sin()[:, :, None]
        z = [y1 * c - y2 * s, y2 * c + y1 * s]
        z = torch.stack(z, -1).flatten(-2) if interleaved else torch.cat(z, -1)
        # the phase is off by at most 2^-32 of a turn (its last bit) and |pos| 2^-65 + |pos f| 2^-53 / 2 pi (the frequency): 2^-20 radians at 2^31
        _close(got, z, R.size(t, pos, rot.inv_freq, interleaved) * 2)


def test_position_zero_is_the_identity(mala):
    q, k = _randn(1, 1, 33, 4, 128), _randn(2, 1, 33, 2, 128)
    qo, ko = mala.rotary(q, k, _rule(mala, 128), positions=torch.zeros((1, 33), dtype=torch.int32, device="cuda"))
    assert torch.equal(qo, q) and torch.equal(ko, k)


def test_there_and_back(mala):
    """The backward pass of the rotation is its inverse."""
    q, k = _randn(1, 1, 50, 4, 64), _randn(2, 1, 50, 2, 64)
    rot = _rule(mala, 64)
    qb, kb, _, _ = mala.rotary_bwd(*mala.rotary(q, k, rot), rot)
    pos = torch.arange(50, device="cuda")[None]
    for t, b in ((q, qb), (k, kb)):
        # two roundings: 2^-8 of each of a pair (turned back: up to sqrt(2) of the sum of the two), and 2^-8 of the value
        assert ((b.double() - t.double()).abs() <= 2.5 * HALF * R.size(t, pos, rot.inv_freq)).all()


def test_columns_behind_pass_through(mala):
    """Infinities and NaN in columns that are not rotated stay where they are; in rotated ones they stay in their pair."""
    q = _randn(3, 1, 4, 2, 80)
    q[0, 1, 0, 50], q[0, 2, 1, 79], q[0, 3, 0, 40] = math.inf, math.nan, -math.inf
    q[0, 0, 1, 3] = math.nan
    for interleaved in (False, True):
        qo, _ = mala.rotary(q, None, _rule(mala, 40, interleaved=interleaved))
        assert torch.equal(qo[..., 40:].nan_to_num(7.0), q[..., 40:].nan_to_num(7.0))
        other = 3 ^ 1 if interleaved else 23
        bad = qo[..., :40].isnan()
        assert bad[0, 0, 1, 3] and bad[0, 0, 1, other] and int(bad.sum()) == 2
    qo, _ = mala.rotary(q, None, _rule(mala, 20))
    assert torch.equal(qo[..., 20:].nan_to_num(7.0), q[..., 20:].nan_to_num(7.0))


def test_in_place_strides_and_queries_alone(mala):
    B, N, Hq, Hkv, d = 2, 37, 4, 2, 128
    rot, norm = _rule(mala, 64), _norm(mala, d, 9)
    x = _randn(4, B, N, Hq + 2 * Hkv, d)
    q, k = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv]
    want = mala.rotary(q, k, rot, norm=norm)
    alone, none = mala.rotary(q, None, rot, norm=norm)
    assert none is None and torch.equal(alone, want[0])
    head_major = q.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(mala.rotary(head_major, k, rot, norm=norm)[0], want[0])
    rest = x[:, :, Hq + Hkv:].clone()
    got = mala.rotary(q, k, rot, norm=norm, q_out=q, k_out=k)
    assert got[0].data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(x[:, :, Hq + Hkv:], rest)
    raw = _randn(5, B, N, Hq + Hkv, d)
    dq, dk = _randn(6, B, N, Hq, d), _randn(7, B, N, Hkv, d)
    want = mala.rotary_bwd(dq, dk, rot, norm=norm, q=raw[:, :, :Hq], k=raw[:, :, Hq:])
    alone = mala.rotary_bwd(dq, None, rot, norm=norm, q=raw[:, :, :Hq])
    assert torch.equal(alone[0], want[0]) and alone[1] is None and alone[3] is None
    got = mala.rotary_bwd(dq, dk, rot, norm=norm, q=raw[:, :, :Hq], k=raw[:, :, Hq:], dq_out=dq, dk_out=dk)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_weights_that_are_not_there(mala):
    """A norm without weights, with one of the two, and without their gradients."""
    d, rot = 64, _rule(mala, 64)
    q, k, dq, dk = (_randn(x, 1, 20, 2, d) for x in range(4))
    ones = torch.ones(d, device="cuda")
    w = _randn(9, d).float()
    full = mala.rotary_bwd(dq, dk, rot, norm=mala.HeadNorm(w, ones), q=q, k=k)
    for norm, has in ((mala.HeadNorm(w, None), (True, False)), (mala.HeadNorm(None, None), (False, False))):
        one = mala.HeadNorm(w if has[0] else ones, ones)
        assert all(torch.equal(a, b) for a, b in zip(mala.rotary(q, k, rot, norm=norm), mala.rotary(q, k, rot, norm=one)))
        got = mala.rotary_bwd(dq, dk, rot, norm=norm, q=q, k=k)
        assert (got[2] is not None, got[3] is not None) == has and torch.equal(got[1], full[1])
    none = mala.rotary_bwd(dq, dk, rot, norm=mala.HeadNorm(w, ones), q=q, k=k, weights=False)
    assert none[2] is None and none[3] is None and torch.equal(none[0], full[0])


def test_rows_of_zeros(mala):
    """A head of zeros: 0 forward (eps > 0), and the gradient 1 / sqrt(eps) of its weighted incoming one."""
    d, rot, norm = 64, _rule(mala, 64), _norm(mala, 64, 2, eps=1e-4)
    q = torch.zeros((1, 3, 2, d), device="cuda", dtype=torch.bfloat16)
    dq = _randn(1, 1, 3, 2, d)
    assert (mala.rotary(q, None, rot, norm=norm)[0] == 0).all()
    got = mala.rotary_bwd(dq, None, rot, norm=norm, q=q)
    pos = torch.arange(3, device="cuda")[None]
    a = _args(rot, norm, 0, pos)
    _close(got[0], R.backward(dq, q, *a)[0], R.backward_size(dq, q, *a))
    assert (got[2] == 0).all()


# ---- packed sequences

@pytest.mark.parametrize("lens_q,lens_k,behind", [([3, 1, 0, 40, 7], None, 0), ([3, 1, 0, 40, 7], [10, 1, 5, 200, 7], 6), ([1], None, 3), ([0, 0, 2], [4, 0, 2], 1),
                                                  ([5] * 300, [9] * 300, 0), ([2, 0, 5] * 220, None, 2), ([2, 0, 5] * 220, [4, 1, 5] * 220, 0)])
@pytest.mark.parametrize("normed", [False, True])
def test_packed(mala, lens_q, lens_k, behind, normed):
    """Bit for bit the single calls; rows behind the last sequence as they are, and without a part in the weights' gradients."""
    Hq, Hkv, d = 4, 2, 64
    rot, norm = _rule(mala, 48), _norm(mala, d, 5) if normed else None
    both = lens_k is not None
    lens_k = lens_k or lens_q
    cu_q, cu_k = ([sum(x[:i]) for i in range(len(x) + 1)] for x in (lens_q, lens_k))
    tq, tk = cu_q[-1] + behind, cu_k[-1] + behind
    q, dq, k, dk = _randn(1, 1, tq, Hq, d), _randn(2, 1, tq, Hq, d), _randn(3, 1, tk, Hkv, d), _randn(4, 1, tk, Hkv, d)
    cq = _i32(cu_q)
    ck = _i32(cu_k) if both else cq
    qo, ko = mala.rotary_varlen(q, k, cq, ck, rot, norm=norm)
    got = mala.rotary_varlen_bwd(dq, dk, cq, ck, rot, norm=norm, q=q, k=k)
    gq, gk, x = (None if r is None else r for r in (0.0, 0.0, None))
    for which, (t, to, g, gx, pos) in enumerate(((q, qo, dq, got[0], R.packed_positions(cu_q, cu_k, tq, True)),
                                                 (k, ko, dk, got[1], R.packed_positions(cu_q, cu_k, tk, False)))):
        have = torch.tensor([p is not None for p in pos], device="cuda")
        p = torch.tensor([p or 0 for p in pos], device="cuda", dtype=torch.int32)[None]
        one, _ = mala.rotary(t, None, rot, positions=p, norm=norm if which == 0 or norm is None else mala.HeadNorm(norm.k_weight, None, norm.eps))
        back = mala.rotary_bwd(g, None, rot, positions=p, norm=norm if which == 0 or norm is None else mala.HeadNorm(norm.k_weight, None, norm.eps), q=t)
        assert torch.equal(to[:, have], one[:, have]) and torch.equal(to[:, ~have], t[:, ~have])
        assert torch.equal(gx[:, have], back[0][:, have]) and torch.equal(gx[:, ~have], g[:, ~have])
        if normed:
            a = _args(rot, norm, which, p[:, have])
            _, dw, total = R.backward(g[:, have], t[:, have], *a)
            _check_dw(got[2 + which], None, dw, total, t.shape[2] + 32)


# ---- gradients through autograd, attention at rotary positions

@pytest.mark.parametrize("normed", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_autograd(mala, normed, packed):
    from paper_2609_32712_b200 import autograd as A
    Hq, Hkv, d = 4, 2, 64
    lens = [5, 1, 30]
    cu = _i32([0, 5, 6, 36])
    B, N = (1, 36) if packed else (2, 19)
    rot = _rule(mala, 64)
    x = _randn(1, B, N, Hq + 2 * Hkv, d)
    leaf = x.clone().requires_grad_(True)
    w = [(_randn(8 + i, d) * 0.2 + 1).requires_grad_(True) for i in range(2)] if normed else [None, None]
    eps = 1e-5 if normed else None
    q, k = leaf[:, :, :Hq], leaf[:, :, Hq:Hq + Hkv]
    if packed:
        qo, ko = A.rotary_packed(q, k, cu, cu, rot, *w, eps=eps)
    else:
        qo, ko = A.rotary(q, k, rot, None, *w, eps=eps)
    a, b = _randn(3, *qo.shape), _randn(4, *ko.shape)
    ((qo * a).sum() + (ko * b).sum()).backward()
    norm = None if not normed else mala.HeadNorm(w[0].detach(), w[1].detach(), eps)
    if packed:
        want = mala.rotary_varlen_bwd(a, b, cu, cu, rot, norm, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv])
    else:
        want = mala.rotary_bwd(a, b, rot, None, norm, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv])
    assert torch.equal(leaf.grad[:, :, :Hq], want[0]) and torch.equal(leaf.grad[:, :, Hq:Hq + Hkv], want[1]) and (leaf.grad[:, :, Hq + Hkv:] == 0).all()
    if normed:
        assert torch.equal(w[0].grad, want[2].to(torch.bfloat16)) and torch.equal(w[1].grad, want[3].to(torch.bfloat16))
    # one output without a gradient, a sum's gradient (a stride of 0)
    leaf.grad = None
    out = A.rotary_packed(q, k, cu, cu, rot, *w, eps=eps) if packed else A.rotary(q, k, rot, None, *w, eps=eps)
    out[0].sum().backward()
    assert torch.isfinite(leaf.grad).all() and (leaf.grad[:, :, Hq:] == 0).all()


@pytest.mark.parametrize("normed", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_attention_at_rotary_positions(mala, normed, packed):
    """mala_attention_rotary is rotary followed by mala_attention, and the gradients those of the two."""
    from paper_2609_32712_b200 import autograd as A
    Hq, Hkv, d, tau = 4, 2, 64, 1e-3
    cu = _i32([0, 150, 151, 400])
    B, N = (1, 400) if packed else (2, 200)
    rot = _rule(mala, 32, magnitude=1.1)
    grads = []
    for fused in (True, False):
        q, k, v = (_randn(s, B, N, h, d).requires_grad_(True) for s, h in ((1, Hq), (2, Hkv), (3, Hkv)))
        w = [(_randn(8 + i, d) * 0.2 + 1).requires_grad_(True) for i in range(2)] if normed else [None, None]
        eps = 1e-5 if normed else None
        if packed:
            args = (cu, cu, 249, 249)
            o = A.mala_attention_rotary_packed(q, k, v, *args, rot, tau, *w, eps=eps) if fused else \
                A.mala_attention_packed(*A.rotary_packed(q, k, cu, cu, rot, *w, eps=eps), v, *args, tau)
        else:
            o = A.mala_attention_rotary(q, k, v, rot, tau, None, *w, eps=eps) if fused else A.mala_attention(*A.rotary(q, k, rot, None, *w, eps=eps), v, tau)
        o.backward(_randn(5, *o.shape))
        grads.append([o.detach()] + [t.grad for t in (q, k, v, *w) if t is not None])
    assert torch.equal(grads[0][0], grads[1][0])
    for a, b in zip(*grads):     # (dQ is added up by atomics: fp32 sums in another order, then one rounding)
        assert ((a.double() - b.double()).norm() <= 2 * HALF * b.double().norm())


def test_a_model_trains_on_it(mala):
    """Projections, normed heads at rotary positions, attention, output projection: against the same in 64 bits, gradients of all weights."""
    from paper_2609_32712_b200 import autograd as A
    N, D, Hq, Hkv, d = 96, 128, 4, 2, 64
    x = _randn(1, 1, N, D)
    w1, w2 = (_randn(2, D, (Hq + 2 * Hkv) * d).float() * D ** -0.5).bfloat16(), (_randn(3, Hq * d, D).float() * (Hq * d) ** -0.5).bfloat16()
    wq, wk = ((_randn(4 + i, d) * 0.2 + 1) for i in range(2))
    rot = _rule(mala, d)
    do = _randn(9, 1, N, D)

    def run(double):
        leaves = [t.detach().to(torch.float64 if double else torch.bfloat16).requires_grad_(True) for t in (w1, w2, wq, wk)]
        xs = x.to(leaves[0].dtype)
        y = (xs @ leaves[0]).view(1, N, Hq + 2 * Hkv, d)
        q, k, v = y.split([Hq, Hkv, Hkv], 2)
        if double:
            pos = torch.arange(N, device="cuda")[None]
            q, k = (R.turn(t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-5) * w, pos, rot.inv_freq) for t, w in ((q, leaves[2]), (k, leaves[3])))
            k, v = (t.repeat_interleave(Hq // Hkv, 2) for t in (k, v))
            s = torch.einsum("bqhd,bkhd->bhqk", q, k) / math.sqrt(d)
            s = s.masked_fill(torch.ones((N, N), dtype=torch.bool, device="cuda").triu(1), -math.inf)
            o = torch.einsum("bhqk,bkhd->bqhd", s.softmax(-1), v)
        else:
            o = A.mala_attention_rotary(q, k, v, rot, 0.0, None, leaves[2], leaves[3], 1e-5)
        (o.reshape(1, N, Hq * d) @ leaves[1]).backward(do.to(leaves[0].dtype))
        return [t.grad.double() for t in leaves]
    for got, want in zip(run(False), run(True)):
        # some ten roundings to bf16 between input and gradient, each 2^-8 at most and independent of one another
        assert (got - want).norm() <= math.sqrt(10) * 2 * HALF * want.norm()


def test_capture_and_streams(mala):
    """Forward and backward captured once and replayed on other inputs, while the same calls run on another stream: bit for bit the eager ones."""
    B, N, Hq, Hkv, d = 1, 300, 8, 2, 128
    rot, norm = _rule(mala, d), _norm(mala, d, 3)
    ins = [_randn(x, B, N, h, d) for x, h in ((1, Hq), (2, Hkv), (3, Hq), (4, Hkv))]
    pos = _i32(list(range(N))).view(1, N)

    def step(q, k, dq, dk):
        return mala.rotary(q, k, rot, positions=pos, norm=norm) + mala.rotary_bwd(dq, dk, rot, positions=pos, norm=norm, q=q, k=k)
    s, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(s):
        step(*ins)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = step(*ins)
    for x in range(3):
        fresh = [_randn(50 + 10 * x + y, *t.shape) for y, t in enumerate(ins)]
        for a, b in zip(ins, fresh):
            a.copy_(b)
        pos.copy_(torch.arange(N, device="cuda")[None] * (x + 1))
        torch.cuda.synchronize()
        with torch.cuda.stream(s2):
            other = step(*fresh)
        graph.replay()
        torch.cuda.synchronize()
        again = step(*ins)
        for a, b, c in zip(out, other, again):
            assert torch.equal(a, b) and torch.equal(a, c)


def test_wrapper_refuses(mala):
    rot = _rule(mala, 64)
    q = _randn(1, 1, 8, 2, 64)
    cu = _i32([0, 8])
    pos = torch.zeros((1, 8), dtype=torch.int32, device="cuda")
    bad = [lambda: mala.rotary(q.float(), None, rot), lambda: mala.rotary(q, q[..., :32], rot), lambda: mala.rotary(q, q, rot, positions=pos.long()),
           lambda: mala.rotary(q, q, rot, positions=pos[:, :4]), lambda: mala.rotary(q.cpu(), None, rot), lambda: mala.rotary(q, q, rot, positions=pos.cpu()),
           lambda: mala.rotary(q, q[:, :4], rot, positions=pos[:, :4]), lambda: mala.rotary(q, None, rot, q_out=q[:, :4]),
           lambda: mala.rotary(q, q, rot, norm=mala.HeadNorm(torch.ones(32, device="cuda"), None)), lambda: mala.rotary(q, q, rot, norm=mala.HeadNorm(torch.ones(64), None)),
           lambda: mala.rotary_bwd(q, q, rot, norm=mala.HeadNorm(None, None)), lambda: mala.rotary_bwd(q, q, rot, norm=mala.HeadNorm(None, None), q=q, k=q[:, :4]),
           lambda: mala.rotary_varlen(q, q, cu.long(), cu, rot), lambda: mala.rotary_varlen(q, q, cu, _i32([0, 4, 8]), rot),
           lambda: mala.rotary_varlen(_randn(1, 2, 8, 2, 64), None, cu, cu, rot)]
    for f in bad:
        with pytest.raises(AssertionError):
            f()
    for f in (lambda: mala.rotary(q, q[:, :4], rot), lambda: mala.rotary(q, None, _rule(mala, 66)), lambda: mala.rotary(q.expand(1, 8, 2, 64)[:, :1].expand(1, 8, 2, 64), None, rot)):
        with pytest.raises(mala.MalaError):
            f()


@pytest.mark.parametrize("attention", [False, True])
def test_changes_before_the_backward_pass_are_noticed(mala, attention):
    """Positions, offsets and frequencies belong to the gradient: changed in place before it is asked for, they raise."""
    from paper_2609_32712_b200 import autograd as A
    for packed in (False, True):
        for which in (0, 1):
            rot = _rule(mala, 64)
            q, k, v = (_randn(x, 1, 40, 2, 64).requires_grad_(True) for x in range(3))
            pos, cu = torch.arange(40, dtype=torch.int32, device="cuda")[None].contiguous(), _i32([0, 15, 40])
            if attention:
                o = A.mala_attention_rotary_packed(q, k, v, cu, cu, 25, 25, rot, 0.0) if packed else A.mala_attention_rotary(q, k, v, rot, 0.0, pos)
            else:
                o = A.rotary_packed(q, k, cu, cu, rot)[0] if packed else A.rotary(q, k, rot, pos)[0]
            (rot.inv_freq if which else cu if packed else pos).add_(1)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                o.sum().backward()


# ---- a serving step

def _pages(seed, fp8, pool, ps, Hkv, d):
    if not fp8:
        return [_randn(seed + x, pool, ps, Hkv, d) for x in range(2)]
    codes = [(_randn(seed + x, pool, ps, Hkv, d).float() * 100).clamp(-448, 448).to(torch.float8_e4m3fn) for x in range(2)]
    return codes + [_randn(seed + 2 + x, pool, Hkv, max(1, ps // 128)).float().abs() * 0.01 + 0.005 for x in range(2)]


def _slots(lens, new, ps, seed, refuse=()):
    """Slots and positions of new rows behind `lens` held ones, the pages of a request anywhere in the pool."""
    g = torch.Generator().manual_seed(seed)
    per = [-(-(a + b) // ps) for a, b in zip(lens, new)]
    order = torch.randperm(sum(per) + 3, generator=g).tolist()
    slots, pos, at = [], [], 0
    for b, (a, n) in enumerate(zip(lens, new)):
        for x in range(a, a + n):
            slots.append(-1 if b in refuse else order[at + x // ps] * ps + x % ps)
            pos.append(x)
        at += per[b]
    return torch.tensor(slots, dtype=torch.int64, device="cuda"), _i32(pos), len(order)


STEPS = [([0, 5, 31, 32, 100], [1] * 5), ([7, 0, 64, 130, 1], [40, 200, 1, 3, 0]), ([1000], [1]), ([0], [513]), ([127, 128, 129, 255], [2, 2, 2, 2])]


@pytest.mark.parametrize("lens,new", STEPS)
@pytest.mark.parametrize("ps,Hq,Hkv,d,rotary,interleaved,normed", [(16, 8, 2, 128, 128, False, False), (128, 6, 3, 64, 64, True, True), (64, 2, 1, 96, 24, False, True),
                                                                   (256, 4, 4, 256, 64, False, False), (8, 4, 1, 80, 40, False, True)])
def test_step_into_bf16_pages(mala, lens, new, ps, Hq, Hkv, d, rotary, interleaved, normed):
    """Bit for bit the rotation followed by the write, and nothing else written."""
    slots, pos, pool = _slots(lens, new, ps, 3, refuse=(2,))
    rows = len(pos)
    rot, norm = _rule(mala, rotary, interleaved=interleaved), _norm(mala, d, 5) if normed else None
    x = _randn(1, rows, Hq + 2 * Hkv, d)
    q, k, v = x.split([Hq, Hkv, Hkv], 1)
    kp, vp = _pages(9, False, pool, ps, Hkv, d)
    want = [kp.clone(), vp.clone()]
    qw, kw = mala.rotary(q[None], k[None], rot, positions=pos[None], norm=norm)
    mala.cache_write(kw[0], v, slots, *want)
    got = mala.rotary_write(q, k, v, pos, slots, kp, vp, rot, norm=norm)
    assert torch.equal(got, qw[0]) and torch.equal(kp, want[0]) and torch.equal(vp, want[1])
    mala.rotary_write(q, k, v, pos, slots, kp, vp, rot, norm=norm, q_out=q)
    assert torch.equal(q, qw[0])


@pytest.mark.parametrize("lens,new", STEPS + [([3] * 90, [1] * 90), ([0, 50, 3000], [6000, 5000, 4000])])
@pytest.mark.parametrize("ps,Hq,Hkv,d,rotary,interleaved,normed", [(16, 8, 2, 128, 128, False, False), (128, 6, 3, 64, 64, True, True), (64, 2, 1, 96, 24, False, True),
                                                                   (256, 4, 4, 128, 64, False, False), (32, 4, 1, 80, 40, False, True), (128, 2, 2, 16, 6, False, False),
                                                                   (64, 4, 2, 128, 32, True, False), (128, 4, 1, 112, 112, False, True)])
def test_step_into_e4m3_pages(mala, lens, new, ps, Hq, Hkv, d, rotary, interleaved, normed):
    """Values: bit for bit cache_write_fp8.  Keys: a unit's scale is its largest rotated magnitude / 448 (or the old scale), good to fp32's
    roundings; new codes are within half a step (2^-4 of the value, or 2^-10 scales where codes are subnormal) of the rotated values in 64 bits, held codes
    on a new scale of theirs, and everything else untouched."""
    slots, pos, pool = _slots(lens, new, ps, 3, refuse=(2,))
    rows = len(pos)
    rot, norm = _rule(mala, rotary, interleaved=interleaved, magnitude=1.1), _norm(mala, d, 5) if normed else None
    x = _randn(1, rows, Hq + 2 * Hkv, d)
    big = torch.rand((rows, 1, 1), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda") < 0.2
    x = torch.where(big, x * 8, x)
    q, k, v = x.split([Hq, Hkv, Hkv], 1)
    kp, vp, ks, vs = _pages(9, True, pool, ps, Hkv, d)
    kp0, ks0 = kp.double(), ks.double()
    want = [t.clone() for t in (kp.view(torch.uint8), vp.view(torch.uint8), ks, vs)]
    mala.cache_write_fp8(k, v, slots, want[0], want[1], want[2], want[3])
    got = mala.rotary_write_fp8(q, k, v, pos, slots, kp, vp, ks, vs, rot, norm=norm)
    assert torch.equal(got, mala.rotary(q[None], None, rot, positions=pos[None], norm=norm)[0][0])
    assert torch.equal(vp.view(torch.uint8), want[1]) and torch.equal(vs, want[3])
    a = _args(rot, norm, 1, pos)
    true, unit = R.forward(k, *a), min(ps, 128)
    ok = slots >= 0
    units, back = torch.unique(slots[ok] // unit, return_inverse=True)
    top = torch.zeros((units.numel(), Hkv), device="cuda", dtype=torch.float64).scatter_reduce_(0, back[:, None].expand(-1, Hkv), true[ok].abs().amax(2), "amax")
    least = torch.full((units.numel(),), unit, device="cuda").scatter_reduce(0, back, slots[ok] % unit, "amin")
    per = ks.shape[2]
    old, now = (t.permute(0, 2, 1).reshape(-1, Hkv)[units] for t in (ks0, ks.double()))
    s = torch.where((least == 0)[:, None], top / 448, torch.maximum(old, top / 448))
    # (the largest value m lies in a pair of length at most sqrt(2) m, so its two terms add up to at most 2 m)
    assert ((now - s).abs() <= 4 * FP32 * s).all()
    codes, before = kp.double().view(-1, Hkv, d), kp0.view(-1, Hkv, d)
    new_codes = codes[slots[ok]]
    x_true, scale = true[ok], now[back][:, :, None]
    err = (new_codes * scale - x_true).abs()
    assert (err <= 2.0 ** -4 * x_true.abs() + 2.0 ** -10 * scale + FP32 * 8 * R.size(k, *a)[ok]).all()
    # keys that the units held
    row = torch.arange(unit, device="cuda")
    held = (row[None] < least[:, None])
    at = (units[:, None] * unit + row[None])[held]
    ratio = (old / now)[:, None].expand(-1, unit, -1)[held][:, :, None]
    moved = before[at] * ratio
    err = (codes[at] - moved).abs()
    assert (err <= torch.where(ratio == 1, torch.zeros_like(ratio), 2.0 ** -4 * moved.abs() + 2.0 ** -10 + 1e-5)).all()
    rest = torch.ones(codes.shape[0], dtype=torch.bool, device="cuda")
    rest[at], rest[slots[ok]] = False, False
    assert torch.equal(codes[rest], before[rest])
    others = torch.ones(pool * per, dtype=torch.bool, device="cuda")
    others[units] = False
    assert torch.equal(ks.permute(0, 2, 1).reshape(-1, Hkv)[others], ks0.float().permute(0, 2, 1).reshape(-1, Hkv)[others])
    assert mala.device_status() == 0


@pytest.mark.parametrize("rotary,interleaved", [(64, False), (24, False), (40, True)])
@pytest.mark.parametrize("lens,new", STEPS)
def test_e4m3_step_at_position_zero_is_the_write(mala, lens, new, rotary, interleaved):
    ps, Hkv, d = 64, 2, 64
    slots, pos, pool = _slots(lens, new, ps, 8)
    k, v, q = _randn(1, len(pos), Hkv, d), _randn(2, len(pos), Hkv, d), _randn(3, len(pos), 4, d)
    a = _pages(9, True, pool, ps, Hkv, d)
    b = [t.clone() for t in a]
    mala.cache_write_fp8(k, v, slots, *a)
    mala.rotary_write_fp8(q, k, v, torch.zeros_like(pos), slots, *b, _rule(mala, rotary, interleaved=interleaved))
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


def test_positions_of_the_tables(mala):
    """page_tables gives the positions of its tokens, 0 where a token has no slot, and everything else as without."""
    for B, new, rows in ((5, [3, 0, 1, 70, 2], 76), (3, [100000, 0, 7], 100010)):
        lens = _i32([5, 0, 31, 8, 2][:B])
        width = 20 if B == 5 else 10
        table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
        for b, n in enumerate(lens.tolist()):
            for x in range(-(-n // 16)):
                table[b, x] = 50 + b * 2 + x
        free = torch.arange(60, dtype=torch.int32, device="cuda")
        a = mala.page_tables(lens, _i32(new), table.clone(), free.clone(), _i32([40]), 16, rows)
        *b, pos = mala.page_tables(lens, _i32(new), table.clone(), free.clone(), _i32([40]), 16, rows, positions=True)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        want = [n + x for n, m in zip(lens.tolist(), new) for x in range(m)] + [0] * rows
        want = [p if s >= 0 else 0 for p, s in zip(want, a[2].tolist())]
        assert pos.tolist() == want and (max(want) > 0)


def test_step_behind_2_to_the_32_bytes(mala):
    """Slots whose pages begin behind 2^32 bytes, bf16 and e4m3."""
    ps, Hkv, d = 128, 1, 128
    pool = 2 ** 32 // (ps * d) + 40                                # e4m3: 4.3 GB
    rot = _rule(mala, d)
    rows = 70
    q, k, v = _randn(1, rows, 2, d), _randn(2, rows, Hkv, d), _randn(3, rows, Hkv, d)
    pos = _i32(list(range(rows)))
    slots = torch.arange(rows, device="cuda") + (pool - 2) * ps
    kp, vp = (torch.zeros((pool, ps, Hkv, d), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.ones((pool, Hkv, 1), device="cuda") for _ in range(2))
    mala.rotary_write_fp8(q, k, v, pos, slots, kp, vp, ks, vs, rot)
    small = [torch.zeros((2, ps, Hkv, d), dtype=torch.uint8, device="cuda") for _ in range(2)] + [torch.ones((2, Hkv, 1), device="cuda") for _ in range(2)]
    mala.rotary_write_fp8(q, k, v, pos, slots - (pool - 2) * ps, *small, rot)
    assert all(torch.equal(a[-2:], b) for a, b in zip((kp, vp, ks, vs), small)) and (small[0] != 0).any()
    b16 = [t.view(torch.bfloat16).view(pool // 2, ps, Hkv, d) for t in (kp, vp)]
    at = slots - (pool - 2) * ps + (pool // 2 - 1) * ps
    mala.rotary_write(q, k, v, pos, at, *b16, rot)
    _, kw = mala.rotary(q[None], k[None], rot)
    assert torch.equal(b16[0][-1, :rows], kw[0]) and torch.equal(b16[1][-1, :rows], v)
