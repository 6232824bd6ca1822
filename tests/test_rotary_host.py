"""CPU checks of the rotary calls, the cache reads and prompts over an e4m3 cache: the plain implementation that the GPU tests compare with is
pinned (differences, relative positions, norms), frequencies and their scalings, and every refusal returns its code without a GPU."""
import ctypes
import math

import pytest
import torch

from tests import rotary_reference as R


@pytest.fixture(scope="module")
def mala():
    from paper_2609_32712_b200 import build, mala as m
    build.build()
    m.lib()
    return m


# ---- the plain implementation

@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("eps", [None, 1e-3])
def test_plain_gradients_by_differences(interleaved, eps):
    g = torch.Generator().manual_seed(1)
    x, dy = (torch.randn((3, 2, 10), generator=g, dtype=torch.float64) for _ in range(2))
    w = torch.randn(10, generator=g, dtype=torch.float64)
    f, pos = torch.rand(3, generator=g, dtype=torch.float64), torch.tensor([0, 5, -9])
    args = (pos, f, interleaved, 1.3, eps, w)
    dx, dw, _ = R.backward(dy, x, *args)
    for t, want in ((x, dx), (w, dw)):
        if want is None:
            continue
        flat = t.view(-1)
        for i in range(flat.numel()):
            at = flat[i].item()
            flat[i] = at + 1e-6
            up = (R.forward(x, *args) * dy).sum()
            flat[i] = at - 1e-6
            down = (R.forward(x, *args) * dy).sum()
            flat[i] = at
            assert abs((up - down).item() / 2e-6 - want.reshape(-1)[i].item()) <= 1e-7


@pytest.mark.parametrize("interleaved", [False, True])
def test_plain_scores_depend_on_the_distance(interleaved):
    g = torch.Generator().manual_seed(2)
    q, k = (torch.randn((1, 1, 16), generator=g, dtype=torch.float64) for _ in range(2))
    f = 100.0 ** (-torch.arange(6, dtype=torch.float64) / 6)
    score = lambda a, b: (R.turn(q, torch.tensor([a]), f, interleaved) * R.turn(k, torch.tensor([b]), f, interleaved)).sum()  # noqa: E731
    assert abs(score(7, 3) - score(1007, 1003)) <= 1e-10 and abs(score(7, 3) - score(8, 3)) > 1e-3
    y = R.turn(q, torch.tensor([12345]), f, interleaved)
    assert torch.equal(y[..., 12:], q[..., 12:]) and abs(y.norm() - q.norm()) <= 1e-12


# ---- frequencies

def test_frequencies(mala):
    f, m = mala.rotary_frequencies(64, 10000.0)
    assert f.dtype is torch.float64 and f.shape == (32,) and m == 1.0 and f[0] == 1 and abs(f[16] - 0.01) <= 1e-15
    assert torch.allclose(mala.rotary_frequencies(64, scaling="linear", factor=4.0)[0], f / 4, rtol=1e-15)
    ntk, _ = mala.rotary_frequencies(64, scaling="ntk", factor=8.0)
    assert ntk[0] == 1 and abs(ntk[-1] / f[-1] * 8 - 1) <= 1e-12 and ((ntk <= f) & (ntk >= f / 8 * (1 - 1e-12))).all()
    assert mala.rotary_frequencies(2, scaling="ntk", factor=8.0)[0].tolist() == [1.0]
    yarn, m = mala.rotary_frequencies(64, scaling="yarn", factor=16.0, original=4096)
    turns = 4096 * f / (2 * math.pi)
    assert abs(m - (0.1 * math.log(16) + 1)) <= 1e-15
    assert torch.equal(yarn[turns > 40], f[turns > 40]) and torch.allclose(yarn[turns < 0.8], f[turns < 0.8] / 16, rtol=1e-12)
    ratio = yarn / f
    assert (ratio[1:] <= ratio[:-1] + 1e-15).all() and ((ratio > 1 / 16 + 1e-3) & (ratio < 1 - 1e-3)).any()
    assert mala.rotary_frequencies(64, scaling="yarn", factor=1.0)[1] == 1.0
    bands, m = mala.rotary_frequencies(64, 500000.0, scaling="bands", factor=8.0, original=8192, low=1.0, high=4.0)
    f = mala.rotary_frequencies(64, 500000.0)[0]
    wave = 2 * math.pi / f
    assert m == 1.0 and torch.equal(bands[wave < 2048], f[wave < 2048]) and torch.allclose(bands[wave > 8192], f[wave > 8192] / 8, rtol=1e-12)
    mid = (wave > 2048) & (wave < 8192)
    part = (8192 / wave[mid] - 1) / 3
    assert mid.any() and torch.allclose(bands[mid], f[mid] / 8 * (1 - part) + f[mid] * part, rtol=1e-12)
    with pytest.raises(ValueError):
        mala.rotary_frequencies(64, scaling="other")
    for bad in (dict(rotary=7), dict(rotary=0), dict(rotary=64, base=-1.0), dict(rotary=64, factor=0.0)):
        with pytest.raises(AssertionError):
            mala.rotary_frequencies(**bad)


def test_objects_refuse(mala):
    for bad in (torch.ones((2, 2)), torch.ones(0), torch.ones(4, dtype=torch.int64)):
        with pytest.raises(AssertionError):
            mala.Rotary(bad, device="cpu")
    r = mala.Rotary(torch.ones(4), interleaved=True, magnitude=2, device="cpu")
    assert r.rotary == 8 and r.inv_freq.dtype is torch.float64 and r.interleaved is True and r.magnitude == 2.0
    w = torch.ones(8)
    for a, b in ((w, w.bfloat16()), (w.half(), None), (w[::2], None), (torch.ones(8, 1), None), (w, torch.ones(16))):
        with pytest.raises(AssertionError):
            mala.HeadNorm(a, b)


# ---- refusals

@pytest.fixture
def args(mala):
    buf = ctypes.create_string_buffer(1 << 20)
    base = (ctypes.addressof(buf) + 255) & ~255
    tin = lambda off=0, sb=4096, sn=256, sh=128, p=True: mala._TIn(base + off if p else None, sb, sn, sh)   # noqa: E731
    tout = lambda off=0, sb=4096, sn=256, sh=128, p=True: mala._TOut(base + off if p else None, sb, sn, sh)  # noqa: E731
    rule = lambda f=base, rotary=128, inter=0, m=1.0: ctypes.byref(mala._Rotary(f, rotary, inter, m))       # noqa: E731
    norm = lambda q=base, k=base, fp32=0, eps=1e-6: ctypes.byref(mala._HeadNorm(q, k, fp32, eps))           # noqa: E731
    return buf, base, tin, tout, rule, norm


INF, NAN = math.inf, math.nan
BAD_RULE = [(dict(f=None), -1), (dict(f="odd"), -3), (dict(rotary=0), -2), (dict(rotary=7), -2), (dict(rotary=130), -2), (dict(rotary=-2), -2),
            (dict(m=0.0), -1), (dict(m=-1.0), -1), (dict(m=INF), -1), (dict(m=NAN), -1)]
BAD_NORM = [(dict(eps=-1.0), -1), (dict(eps=NAN), -1), (dict(eps=INF), -1), (dict(q="odd"), -3), (dict(k="odd"), -3), (dict(k="odd2", fp32=1), -3)]


@pytest.mark.parametrize("kw,code", BAD_RULE + BAD_NORM)
def test_rule_and_norm_are_refused(mala, args, kw, code):
    buf, base, tin, tout, rule, norm = args
    kw = {a: base + (1 if b == "odd" else 2) if b in ("odd", "odd2") else b for a, b in kw.items()}
    r = rule(**{a: b for a, b in kw.items() if a in ("f", "rotary", "inter", "m")})
    n = norm(**{a: b for a, b in kw.items() if a in ("q", "k", "fp32", "eps")})
    L = mala.lib()
    assert L.mala_rotary_fwd(tin(), tin(), None, r, n, tout(), tout(), 1, 4, 4, 2, 2, 128, None) == code
    assert L.mala_rotary_bwd(tin(), tin(), tin(), tin(), None, r, n, tout(), tout(), None, None, 1, 4, 4, 2, 2, 128, None, 0, None) == code
    assert L.mala_rotary_fwd_varlen(tin(), tin(), base, base, r, n, tout(), tout(), 1, 2, 2, 4, 4, 128, None) == code
    assert L.mala_rotary_bwd_varlen(tin(), tin(), tin(), tin(), base, base, r, n, tout(), tout(), None, None, 1, 2, 2, 4, 4, 128, None, 0, None) == code
    assert L.mala_rotary_write(tin(), tin(), tin(), base, base, r, n, tout(), tout(), tout(), 4, 2, 2, 4, 16, 128, None) == code
    assert L.mala_rotary_write_fp8(tin(), tin(), tin(), base, base, r, n, tout(), tout(), tout(), base, base, 4, 2, 2, 4, 16, 128, None) == code


def test_rotary_calls_are_refused(mala, args):
    buf, base, tin, tout, rule, norm = args
    L = mala.lib()

    def fwd(q=None, k=None, pos=None, n=None, qo=None, ko=None, B=1, Nq=4, Nk=4, Hq=2, Hkv=2, d=128, rotary=8):
        return L.mala_rotary_fwd(q or tin(), k or tin(), pos, rule(rotary=rotary), n, qo or tout(), ko or tout(), B, Nq, Nk, Hq, Hkv, d, None)
    for kw, code in [(dict(B=0), -1), (dict(Nq=0), -1), (dict(Nk=0), -1), (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(Nq=5), -2), (dict(d=0), -1), (dict(d=12), -2),
                     (dict(d=264), -2), (dict(Hq=65536), -2), (dict(Hkv=65536), -2), (dict(B=1 << 20, Nq=2000, Nk=2000), -2), (dict(pos=base + 2), -3),
                     (dict(q=tin(p=False)), -1), (dict(k=tin(p=False)), -1), (dict(qo=tout(p=False)), -1), (dict(ko=tout(p=False)), -1), (dict(q=tin(8)), -3),
                     (dict(k=tin(2)), -3), (dict(qo=tout(8)), -3), (dict(ko=tout(8)), -3), (dict(q=tin(sn=0)), -1), (dict(q=tin(sn=-256)), -1), (dict(q=tin(sh=0)), -1),
                     (dict(k=tin(sn=129)), -3), (dict(k=tin(sh=4)), -3), (dict(qo=tout(sn=0)), -1), (dict(ko=tout(sh=12)), -3),
                     (dict(B=2, q=tin(sb=0)), -1), (dict(B=2, ko=tout(sb=4)), -3)]:
        assert fwd(**kw) == code, kw
    none = dict(k=mala._TIn(None, 0, 0, 0), ko=mala._TOut(None, 0, 0, 0), Hkv=0)
    assert fwd(**none, d=12) == -2 and fwd(k=mala._TIn(None, 0, 0, 0)) == -1

    def bwd(n=None, q=None, k=None, dwq=None, dwk=None, ws=None, nbytes=0, d=128, dq=None, dk=None, dko=None):
        return L.mala_rotary_bwd(dq or tin(), dk or tin(), q or tin(), k or tin(), None, rule(rotary=8), n, tout(), dko or tout(), dwq, dwk, 1, 4, 4, 2, 2, d,
                                 ws, nbytes, None)
    big = mala.lib().mala_rotary_workspace_bytes(128)
    for kw, code in [(dict(dwq=base), -1), (dict(dwk=base), -1), (dict(n=norm(), dwq=base), -1), (dict(n=norm(), dwq=base, ws=base + 16, nbytes=big), -3),
                     (dict(n=norm(), dwq=base, ws=base, nbytes=big - 1), -4), (dict(n=norm(q=None), dwq=base, ws=base, nbytes=big), -1),
                     (dict(n=norm(k=None), dwk=base, ws=base, nbytes=big), -1), (dict(n=norm(), dwk=base + 2, ws=base, nbytes=big), -3),
                     (dict(n=norm(), q=mala._TIn(None, 0, 0, 0)), -1), (dict(n=norm(), k=mala._TIn(None, 0, 0, 0)), -1), (dict(n=norm(), q=tin(8)), -3), (dict(n=norm(), k=tin(sh=4)), -3),
                     (dict(n=norm(), dk=mala._TIn(None, 0, 0, 0)), -1), (dict(n=norm(), dk=mala._TIn(None, 0, 0, 0), dko=mala._TOut(None, 0, 0, 0), dwk=base, ws=base, nbytes=big), -1), (dict(d=20), -2)]:
        assert bwd(**kw) == code, kw
    assert [mala.lib().mala_rotary_workspace_bytes(x) for x in (0, -8, 12, 264)] == [0] * 4 and big > 0
    for cu_q, cu_k, B, code in [(None, base, 1, -1), (base, None, 1, -1), (base, base, 0, -1), (base + 2, base, 1, -3), (base, base + 1, 1, -3)]:
        assert L.mala_rotary_fwd_varlen(tin(), tin(), cu_q, cu_k, rule(rotary=8), None, tout(), tout(), B, 2, 2, 4, 4, 128, None) == code
        assert L.mala_rotary_bwd_varlen(tin(), tin(), tin(), tin(), cu_q, cu_k, rule(rotary=8), None, tout(), tout(), None, None, B, 2, 2, 4, 4, 128, None, 0,
                                        None) == code


def test_step_calls_are_refused(mala, args):
    buf, base, tin, tout, rule, norm = args
    L = mala.lib()

    def step(fp8, q=None, k=None, v=None, pos=base, slots=base, qo=None, kp=None, vp=None, ks=base, vs=base, rows=4, Hq=2, Hkv=2, pages=4, ps=16, d=128):
        a = (q or tin(), k or tin(), v or tin(), pos, slots, rule(rotary=8), None, qo or tout(), kp or tout(), vp or tout())
        a += (ks, vs) if fp8 else ()
        return (L.mala_rotary_write_fp8 if fp8 else L.mala_rotary_write)(*a, rows, Hq, Hkv, pages, ps, d, None)
    for kw, code in [(dict(rows=-1), -1), (dict(rows=0), 0), (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(Hq=65536), -2), (dict(pages=0), -1), (dict(ps=0), -1),
                     (dict(ps=12), -2), (dict(ps=192), -2), (dict(ps=4), -2), (dict(d=0), -1), (dict(d=12), -2), (dict(d=264), -2), (dict(rows=(1 << 30) + 1), -2),
                     (dict(pos=None), -1), (dict(pos=base + 2), -3), (dict(slots=None), -1), (dict(slots=base + 4), -3), (dict(q=tin(p=False)), -1),
                     (dict(k=tin(p=False)), -1), (dict(v=tin(p=False)), -1), (dict(qo=tout(p=False)), -1), (dict(kp=tout(p=False)), -1), (dict(vp=tout(8)), -3),
                     (dict(q=tin(sn=0)), -1), (dict(qo=tout(sh=0)), -1), (dict(q=tin(sh=12)), -3), (dict(k=tin(sn=12)), -3), (dict(kp=tout(sn=0)), -1)]:
        for fp8 in (False, True):
            assert step(fp8, **kw) == code, (kw, fp8)
    for kw, code in [(dict(ks=None), -1), (dict(vs=None), -1), (dict(ks=base + 1), -3), (dict(vs=base + 2), -3), (dict(d=136), -2), (dict(d=24), -2), (dict(ps=8), -2)]:
        assert step(True, **kw) == code, kw


def test_reads_are_refused(mala, args):
    buf, base, tin, tout, rule, norm = args
    L = mala.lib()

    def read(fp8, kp=None, vp=None, ks=base, vs=base, table=base, lens=base, k=None, v=None, cu=base + 4096, B=2, Hkv=2, pages=4, ps=16, most=4, rows=8, d=128):
        a = (kp or tin(), vp or tin()) + ((ks, vs) if fp8 else ()) + (table, lens, k or tout(), v or tout(), cu, B, Hkv, pages, ps, most, rows, d, None)
        return (L.mala_cache_read_fp8 if fp8 else L.mala_cache_read)(*a)
    for kw, code in [(dict(B=0), -1), (dict(Hkv=0), -1), (dict(pages=0), -1), (dict(ps=0), -1), (dict(most=0), -1), (dict(rows=-1), -1), (dict(d=0), -1), (dict(ps=12), -2),
                     (dict(B=16385), -2), (dict(Hkv=65536), -2), (dict(rows=(1 << 30) + 1), -2), (dict(most=1 << 30), -2), (dict(d=12), -2), (dict(d=264), -2),
                     (dict(table=None), -1), (dict(lens=None), -1), (dict(cu=None), -1), (dict(cu=base), -1), (dict(table=base + 2), -3), (dict(lens=base + 1), -3),
                     (dict(cu=base + 4097), -3), (dict(kp=tin(p=False)), -1), (dict(vp=tin(8)), -3), (dict(k=tout(p=False)), -1), (dict(v=tout(8)), -3),
                     (dict(kp=tin(sn=0)), -1), (dict(k=tout(sn=0)), -1), (dict(v=tout(sh=12)), -3), (dict(vp=tin(sh=12)), -3)]:
        for fp8 in (False, True):
            assert read(fp8, **kw) == code, (kw, fp8)
    for kw, code in [(dict(ks=None), -1), (dict(vs=base + 1), -3), (dict(d=136), -2), (dict(d=24), -2), (dict(ps=8), -2)]:
        assert read(True, **kw) == code, kw


def test_paged_fp8_is_refused(mala, args):
    buf, base, tin, tout, rule, norm = args
    L = mala.lib()
    need = L.mala_paged_fp8_workspace_bytes(2, 2, 64, 128)
    assert need == 2 * 64 * 2 * 128 * 2 + 768 + 256      # (three blocks of 24 scales for each of two heads)
    assert [L.mala_paged_fp8_workspace_bytes(*a) for a in ((0, 2, 64, 128), (2, 0, 64, 128), (2, 2, 0, 128), (2, 2, 64, 24), (2, 2, 64, 256), (2, 2, 64, 0))] == [0] * 6

    def call(q=None, kp=None, vp=None, ks=base, vs=base, cu=base, table=base, lens=base, o=None, lse=base, B=2, Hq=4, Hkv=2, total_q=8, most_q=8, total_k=64, pages=4,
             ps=16, most=4, d=128, causal=1, scale=0.1, tau=0.0, ws=base, nbytes=need):
        return L.mala_fwd_paged_fp8(q or tin(), kp or tin(), vp or tin(), ks, vs, cu, table, lens, o or tout(), lse, None, B, Hq, Hkv, total_q, most_q, total_k, pages,
                                    ps, most, d, causal, scale, tau, ws, nbytes, None)
    for kw, code in [(dict(cu=None), -1), (dict(table=None), -1), (dict(lens=None), -1), (dict(lse=None), -1), (dict(ws=None), -1), (dict(ws=base + 16), -3),
                     (dict(nbytes=need - 1), -4), (dict(ks=None), -1), (dict(vs=base + 2), -3), (dict(B=0), -1), (dict(Hq=3), -2), (dict(total_q=0), -1),
                     (dict(most_q=9), -2), (dict(total_k=0), -1), (dict(total_k=7), -2), (dict(pages=0), -1), (dict(ps=8), -2), (dict(ps=24), -2), (dict(most=0), -1),
                     (dict(d=136), -2), (dict(d=24), -2), (dict(scale=0.0), -1), (dict(tau=-1.0), -1), (dict(tau=NAN), -1), (dict(q=tin(8)), -3), (dict(o=tout(p=False)), -1),
                     (dict(kp=tin(p=False)), -1), (dict(vp=tin(sn=8)), -3), (dict(cu=base + 2), -3), (dict(table=base + 2), -3), (dict(lens=base + 2), -3),
                     (dict(B=20000, ws=base, nbytes=1 << 40), -2)]:
        assert call(**kw) == code, kw


def test_positions_of_the_tables_are_refused(mala, args):
    buf, base, *_ = args
    f = mala.lib().mala_page_tables_positions
    at = [base + 512 * x for x in range(10)]

    def call(pos, rows=4, B=2):
        return f(at[0], at[1], at[2], at[3], at[4], at[5], at[6], at[7], pos, at[9], B, 4, 16, 8, rows, None)
    assert call(None) == -1 and call(at[8] + 2) == -3 and call(at[0]) == -1 and call(at[1]) == -1 and call(at[8], B=0) == -1


def test_autograd_entry_points_refuse(mala):
    from paper_2609_32712_b200 import autograd as A
    r = mala.Rotary(torch.ones(4), device="cpu")
    q = torch.zeros((1, 4, 2, 16), dtype=torch.bfloat16)
    w = torch.ones(16)
    for f in (lambda: A.rotary(q, q, r, q_weight=w), lambda: A.mala_attention_rotary(q, q, q, r, 0.0, k_weight=w),
              lambda: A.rotary_packed(q, q, None, None, r, q_weight=w), lambda: A.mala_attention_rotary_packed(q, q, q, None, None, 4, 4, r, 0.0, q_weight=w)):
        with pytest.raises(AssertionError):
            f()


def test_suggested_ranges(mala):
    f = mala.lib().mala_paged_fp8_suggest_splits
    for bad in ((0, 8, 1, 1, 1), (1, 0, 1, 1, 1), (1, 8, 0, 1, 1), (1, 8, 1, 0, 1), (1, 8, 1, 1, 0)):
        assert f(*bad, 148) == -1
    assert f(1, 32, 2048, 30000, 30000, 148) == 1                                # as many CTAs as fill the SMs
    assert f(1, 8, 20, 8000, 8000, 148) == 9                                     # 16 blocks of queries
    assert f(1, 8, 20, 100, 100, 148) == 1                                       # one key block
    assert 2 <= f(1, 1, 1, 2 ** 31 - 1, 2 ** 31 - 1, 148) <= 32
    assert f(65535, 8, 1, 8000, 8000, 148) == 1                                  # (the grid's third coordinate)
    need, split = mala.lib().mala_paged_fp8_workspace_bytes, mala.lib().mala_paged_fp8_split_workspace_bytes
    assert split(2, 4, 2, 40, 64, 128, 1) == need(2, 2, 64, 128)
    assert split(2, 4, 2, 40, 64, 100, 3) == 0 and split(2, 4, 2, 0, 64, 128, 3) == 0 and split(2, 4, 2, 40, 64, 128, 0) == 0
    assert split(2, 4, 2, 40, 64, 96, 3) == need(2, 2, 64, 96) + 2 * 4 * 3 * 40 * (128 + 1) * 4
