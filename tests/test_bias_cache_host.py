"""CPU checks of the calls with a relative position bias and of those that fill a paged cache: the plain implementation that the
GPU tests compare with is pinned (buckets, softmax, gradients by differences), and every refusal returns its code without a GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

from tests import bias_reference as R


@pytest.fixture(scope="module")
def mala():
    from paper_2609_32712_b200 import build, mala as m
    build.build()
    m.lib()
    return m


# ---- the plain implementation

@pytest.mark.parametrize("nb,md,bidir", [(32, 128, False), (32, 128, True), (7, 50, False), (4, 2, True), (2, 65536, False), (128, 4000, False), (24, 768, True)])
def test_buckets(nb, md, bidir):
    """Against the logarithms in the formula, away from its borders, and by their properties."""
    delta = torch.arange(-5000, 5001)
    b = R.buckets(delta, nb, md, bidir)
    h = nb // 2 if bidir else nb
    e = h // 2
    for d in range(-5000, 5001, 7):
        n = abs(d) if bidir else max(-d, 0)
        side = h if bidir and d > 0 else 0
        if n < e:
            want = n
        else:
            x = (h - e) * math.log(n / e) / math.log(md / e)
            if abs(x - round(x)) < 1e-9 and n < md:
                # a border: the bucket that begins there, exactly
                assert n ** (h - e) * e ** round(x) == md ** round(x) * e ** (h - e)
                x = round(x)
            want = min(h - 1, e + math.floor(x))
        assert int(b[d + 5000]) == side + want, d
    assert int(b.min()) >= 0 and int(b.max()) < nb
    before = b[:5001].flip(0)                       # distances 0 .. 5000
    assert (before[1:] >= before[:-1]).all() and (before[md:] == h - 1).all()
    if not bidir:
        assert (b[5001:] == 0).all()


def test_plain_attention_by_differences():
    """The reference's gradients against central differences of its forward, the table's among them, with shared buckets and
    masked ones."""
    g = torch.Generator().manual_seed(3)
    Nq, Nk, d, nb, md = 9, 13, 6, 8, 7
    for causal, bidir in ((True, False), (False, True), (True, True)):
        q, k, v, do, table = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((Nq, d), (Nk, d), (Nk, d), (Nq, d), (nb,)))
        r = R.head(q, k, v, table, do, 0.3, nb, md, bidir, causal)
        f = lambda: (R.head(q, k, v, table, None, 0.3, nb, md, bidir, causal)["o"] * do).sum()  # noqa: B023,E731
        for t, name in ((q, "dq"), (k, "dk"), (v, "dv"), (table, "dtable")):
            flat, want = t.view(-1), r[name].reshape(-1)
            for x in range(0, flat.numel(), 3 if flat.numel() > 20 else 1):
                at, h = flat[x].item(), 1e-5
                flat[x] = at + h
                up = f()
                flat[x] = at - h
                down = f()
                flat[x] = at
                assert abs((up - down).item() / (2 * h) - want[x].item()) <= 1e-8


def test_plain_attention_masks():
    """A bucket of -inf is as if its keys were not there; a row of nothing else is empty."""
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn((7, 4), generator=g, dtype=torch.float64) for _ in range(3))
    table = torch.zeros(8, dtype=torch.float64)
    table[0] = -math.inf
    r = R.head(q, k, v, table, v, 1.0, 8, 20, False, True)
    assert (r["o"][0] == 0).all() and r["lse"][0] == -math.inf and (r["dq"][0] == 0).all()
    for i in range(1, 7):
        s = q[i] @ k[:i].T
        assert torch.allclose(r["o"][i], torch.softmax(s, 0) @ v[:i], atol=1e-12) and torch.allclose(r["lse"][i], torch.logsumexp(s, 0))


# ---- refusals

@pytest.fixture
def args(mala):
    buf = ctypes.create_string_buffer(1 << 22)
    base = (ctypes.addressof(buf) + 255) & ~255
    tin = lambda off=0, sn=256: mala._TIn(base + off, 1024, sn, 128)   # noqa: E731
    tout = lambda off=0, sn=256: mala._TOut(base + off, 1024, sn, 128)  # noqa: E731
    return buf, base, tin, tout


def _bias(mala, base, **kw):
    return mala._RelBias(kw.get("table", base), kw.get("sb", 2), kw.get("nb", 32), kw.get("md", 128), kw.get("bidir", 0))


BAD_BIAS = [(dict(table=None), -1), (dict(table="odd"), -3), (dict(sb=-1), -1), (dict(nb=1), -2), (dict(nb=129), -2), (dict(nb=0), -2),
            (dict(nb=33, bidir=1), -2), (dict(nb=2, bidir=1), -2), (dict(md=16), -2), (dict(md=65537), -2), (dict(md=-5), -2)]


@pytest.mark.parametrize("kw,code", BAD_BIAS)
def test_bias_is_refused(mala, args, kw, code):
    buf, base, tin, tout = args
    if kw.get("table") == "odd":
        kw = dict(kw, table=base + 1)
    b = ctypes.byref(_bias(mala, base, **kw))
    L = mala.lib()
    assert L.mala_fwd_bias(tin(), tin(), tin(), b, tout(), base, None, 1, 2, 2, 4, 4, 128, 1, 0.1, 0.0, base, 1 << 21, None) == code
    assert L.mala_bwd_bias(tin(), tin(), tin(), tin(), tin(), base, b, tout(), tout(), tout(), base, 2, None, 1, 2, 2, 4, 4, 128, 1, 0.1, 0.0,
                           base, 1 << 21, None) == code
    assert L.mala_fwd_varlen_bias(tin(), tin(), tin(), base, base, b, tout(), base, None, 1, 2, 2, 4, 4, 4, 4, 128, 1, 0.1, 0.0, base, 1 << 21,
                                  None) == code
    assert L.mala_decode_paged_bias(tin(), tin(), tin(), base, base, b, tout(), None, None, 1, 2, 2, 4, 16, 4, 1, 128, 0.1, 0.0, 2, base, 1 << 21,
                                    None) == code


def test_bias_calls_refuse(mala, args):
    buf, base, tin, tout = args
    L = mala.lib()
    b = ctypes.byref(_bias(mala, base))
    f = lambda **kw: L.mala_fwd_bias(kw.get("q", tin()), tin(), tin(), kw.get("bias", b), tout(), kw.get("lse", base), None, 1,   # noqa: E731
                                     kw.get("Hq", 2), 2, kw.get("Nq", 4), kw.get("Nk", 4), kw.get("d", 128), kw.get("causal", 1),
                                     kw.get("scale", 0.1), kw.get("tau", 0.0), kw.get("ws", base), kw.get("n", 1 << 21), None)
    assert f(bias=None) == -1 and f(lse=None) == -1 and f(ws=None) == -1 and f(scale=0.0) == -1 and f(tau=-1.0) == -1
    assert f(d=136) == -2 and f(d=256) == -2 and f(d=12) == -2 and f(Hq=3) == -2 and f(Nq=5) == -2
    assert f(ws=base + 16) == -3 and f(q=tin(off=2)) == -3 and f(n=100) == -4
    h = lambda **kw: L.mala_bwd_bias(tin(), tin(), tin(), tin(), tin(), base, kw.get("bias", b), tout(), tout(), tout(), kw.get("dt", base),   # noqa: E731
                                     kw.get("sb", 2), None, 1, 2, 2, 4, 4, 128, 1, 0.1, 0.0, base, kw.get("n", 1 << 21), None)
    assert h(bias=None) == -1 and h(dt=None) == -1 and h(sb=1) == -1 and h(dt=base + 1) == -3 and h(n=1 << 10) == -4
    need = int(L.mala_bias_workspace_bytes(mala.OP_BWD, 1, 2, 2, 4, 4, 0, 128, 0, 32, 128))
    assert need < 1 << 21
    if not torch.cuda.is_available():       # valid arguments on a machine without a GPU: a loud CUDA error
        assert h(n=need) in (-5, -6) and f() in (-5, -6)
    v = lambda **kw: L.mala_bwd_varlen_bias(tin(), tin(), tin(), tin(), tin(), base, kw.get("cq", base), kw.get("ck", base), b, tout(), tout(),   # noqa: E731
                                            tout(), base, 2, None, 2, 2, 2, 8, 8, kw.get("mq", 4), kw.get("mk", 4), 128, 1, 0.1, 0.0, base, 1 << 21, None)
    assert v(cq=None) == -1 and v(ck=None) == -1 and v(mq=0) == -1 and v(mq=9) == -2 and v(mq=5, mk=4) == -2
    dec = lambda **kw: L.mala_decode_paged_bias(tin(), tin(), tin(), kw.get("bt", base), base, kw.get("bias", b), tout(), None, None, 1,   # noqa: E731
                                                kw.get("Hq", 2), 2, 4, kw.get("ps", 16), 4, kw.get("Sq", 1), kw.get("d", 128), 0.1, 0.0,
                                                kw.get("S", 2), base, kw.get("n", 1 << 21), None)
    assert dec(bt=None) == -1 and dec(bias=None) == -1 and dec(S=0) == -1 and dec(ps=24) == -2 and dec(Sq=17) == -2 and dec(d=256) == -2
    assert dec(n=2048) == -4
    for bad in ((3, 1, 2, 2, 4, 4, 0, 128, 0, 32, 128), (0, 0, 2, 2, 4, 4, 0, 128, 0, 32, 128), (0, 1, 2, 2, 4, 4, 0, 200, 0, 32, 128),
                (0, 1, 2, 2, 4, 4, 0, 128, 0, 200, 128), (0, 1, 2, 2, 4, 4, 0, 128, 0, 32, 1 << 17), (2, 1, 2, 2, 1, 4, 0, 128, 0, 32, 128)):
        assert L.mala_bias_workspace_bytes(*bad) == 0


def test_table_calls_refuse(mala, args):
    buf, base, tin, tout = args
    L = mala.lib()
    at = lambda x: base + 4096 * x  # noqa: E731
    names = ("seqlens", "new", "table", "free", "count", "cu", "lens", "slots", "left")

    def tables(B=2, mp=4, ps=16, np_=8, rows=4, **kw):
        a = [kw.get(n, at(x)) for x, n in enumerate(names)]
        return L.mala_page_tables(*a, B, mp, ps, np_, rows, None)
    for n in names:
        assert tables(**{n: None}) == -1 and tables(**{n: at(20) + (4 if n == "slots" else 2)}) == -3
    assert tables(lens=at(0)) == -1 and tables(left=at(4)) == -1 and tables(cu=at(0)) == -1 and tables(cu=at(1)) == -1 and tables(lens=at(1)) == -1
    assert tables(B=0) == -1 and tables(mp=0) == -1 and tables(ps=0) == -1 and tables(np_=0) == -1 and tables(rows=-1) == -1
    assert tables(B=16385) == -2 and tables(ps=24) == -2 and tables(ps=4) == -2 and tables(ps=130) == -2 and tables(mp=1 << 28) == -2
    assert tables(rows=(1 << 30) + 1) == -2 and tables(B=16384, mp=1 << 17, ps=8) == -2

    def release(B=2, mp=4, ps=16, np_=8, **kw):
        a = [kw.get(n, at(x)) for x, n in enumerate(("done", "seqlens", "table", "free", "count", "lens", "left"))]
        return L.mala_release_pages(*a, B, mp, ps, np_, None)
    for n in ("done", "seqlens", "table", "free", "count", "lens", "left"):
        assert release(**{n: None}) == -1
    assert release(lens=at(1)) == -1 and release(left=at(4)) == -1 and release(B=16385) == -2 and release(ps=100) == -2 and release(free=base + 2) == -3


def test_cache_writes_refuse(mala, args):
    buf, base, tin, tout = args
    L = mala.lib()
    w = lambda **kw: L.mala_cache_write(kw.get("k", tin()), tin(), kw.get("s", base), kw.get("kp", tout()), tout(), kw.get("rows", 4), 2,   # noqa: E731
                                        kw.get("np", 4), kw.get("ps", 16), kw.get("d", 128), None)
    assert w(s=None) == -1 and w(rows=-1) == -1 and w(np=0) == -1 and w(ps=0) == -1 and w(d=0) == -1 and w(k=mala._TIn(None, 0, 256, 128)) == -1
    assert w(kp=mala._TOut(base, 0, 256, 128)) == -1
    assert w(ps=24) == -2 and w(d=12) == -2 and w(d=264) == -2 and w(rows=(1 << 30) + 1) == -2
    assert w(s=base + 4) == -3 and w(k=tin(off=8)) == -3 and w(k=tin(sn=130)) == -3 and w(kp=tout(off=8)) == -3
    assert w(rows=0) == 0 and w(rows=0, s=None) == 0           # (nothing to do, also without a GPU)
    z = lambda **kw: L.mala_cache_write_fp8(tin(), tin(), base, kw.get("kp", tout()), tout(), kw.get("ks", base), kw.get("vs", base), kw.get("rows", 4),   # noqa: E731
                                            2, 4, kw.get("ps", 16), kw.get("d", 128), None)
    assert z(ks=None) == -1 and z(vs=None) == -1 and z(ps=8) == -2 and z(d=24) == -2 and z(d=144) == -2 and z(rows=(1 << 30) + 1) == -2
    assert z(ks=base + 2) == -3 and z(kp=mala._TOut(base, 1024, 264, 128)) == -3
    assert z(rows=0) == 0


def test_python_checks(mala):
    with pytest.raises(AssertionError):
        mala.RelativeBias(torch.zeros(32, 4))
    with pytest.raises(AssertionError):
        mala.RelativeBias(torch.zeros(4, 32, dtype=torch.bfloat16).t())
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(AssertionError):
        mala.page_tables(i.long(), i, torch.zeros(4, 2, dtype=torch.int32), i, i[:1], 16, 4)
    with pytest.raises(AssertionError):
        mala.cache_write(torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 64, dtype=torch.bfloat16), i, None, None)
    b16 = lambda *n: torch.zeros(n, dtype=torch.bfloat16)   # noqa: E731
    q, k, bias = b16(1, 4, 2, 64), b16(1, 6, 2, 64), mala.RelativeBias(b16(32, 2))
    lse = torch.zeros(1, 2, 4)
    for bad in (lambda: mala.fwd_bias(q, k, k[:, :5], bias, 0.1, 0.0), lambda: mala.fwd_bias(q, k, k, bias, 0.1, 0.0, lse=lse[:, :, :3]),
                lambda: mala.fwd_bias(q, k, k, bias, 0.1, 0.0, out=q[:, :3]), lambda: mala.bwd_bias(q, k, k, q, q[:, :3], lse, bias, 0.1, 0.0),
                lambda: mala.bwd_bias(q, k, k, q, q, lse.double(), bias, 0.1, 0.0), lambda: mala.bwd_bias(q, k, k, q, q, lse, bias, 0.1, 0.0, dk=q),
                lambda: mala.fwd_varlen_bias(q, k, k[:, :3], i[:2], i[:2], 4, 6, bias, 0.1, 0.0),
                lambda: mala.bwd_varlen_bias(q, k, k, q, q, lse, i[:2], i[:2], 4, 6, bias, 0.1, 0.0),
                lambda: mala.decode_paged_bias(q, b16(3, 16, 2, 64), b16(2, 16, 2, 64), i[:2].view(1, 2), i[:1], bias, 0.1, 0.0, 2),
                lambda: mala.page_tables(i, i, torch.zeros(4, 2, dtype=torch.int32), i, i[:0], 16, 4),
                lambda: mala.release_pages(i > 0, i, torch.zeros(4, 2, dtype=torch.int32), i, i[:2], 16)):
        with pytest.raises(AssertionError):
            bad()


# ---- where the buckets begin, as the kernels have it

def test_starts_of_the_buckets(tmp_path):
    """The library's own function against whole-number powers: every number of buckets with the distances up to 1500 and a spread of larger
    ones, and pairs where a bucket begins less than 1e-9 above a whole number."""
    import os
    import subprocess
    here = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_32712_b200", "csrc")
    src = tmp_path / "starts.cpp"
    src.write_text('#include "mala_bias_starts.h"\nextern "C" int starts(int nb, int md, int bidir, int* out) { mala::BiasStarts s; if '
                   '(!mala::bias_starts(nb, md, bidir, &s)) return -1; for (int i = 0; i < s.count; ++i) out[i] = s.first[i]; out[s.count] = s.reach; '
                   'return s.count; }\n')
    so = tmp_path / "starts.so"
    subprocess.check_call(["g++", "-O2", "-shared", "-fPIC", f"-I{here}", str(src), "-o", str(so)])
    f = ctypes.CDLL(str(so)).starts
    out = (ctypes.c_int * 129)()

    def check(nb, md, bidir):
        e, h, want = R.bucket_starts(nb, md, bidir)
        assert f(nb, md, int(bidir), out) == len(want)
        assert list(out[:len(want)]) == want, (nb, md, bidir)
        assert out[len(want)] == (want[-1] if want else e)
    named = [(73, 905), (64, 21228), (32, 43921)]
    for nb, md in named:
        check(nb, md, False)
    for nb in range(2, 129):
        e = nb // 2
        dists = np.concatenate([np.arange(e + 1, 1501), np.unique(np.geomspace(1501, 65536, 60).astype(int)), [2 ** x for x in range(11, 17)]])
        w = nb - e
        x = e * np.exp(np.arange(1, w)[:, None] * np.log(dists / e) / w)
        near = (np.abs(x - np.rint(x)) < 1e-8 * x).any(0)      # (elsewhere the ceiling is beyond doubt)
        assert f(nb, 65536, 0, out) == w - 1
        for md, c, is_near in zip(dists.tolist(), np.ceil(x).T.astype(int).tolist(), near.tolist()):
            if is_near:
                check(nb, md, False)
            else:
                assert f(nb, md, 0, out) == w - 1 and list(out[:w - 1]) == c, (nb, md)
    for nb, md in ((4, 2), (32, 128), (24, 768), (128, 65536), (128, 40)):
        check(nb, md, True)
    for bad in ((1, 128, 0), (129, 128, 0), (33, 128, 1), (2, 128, 1), (32, 16, 0), (32, 65537, 0), (32, 0, 0)):
        assert f(*bad, out) == -1


def test_workspace_sizes_beyond_32_bits(mala):
    """Rows that do not count in 32 bits have no workspace; the largest ones that do have one that grows as it should."""
    f = mala.lib().mala_bias_workspace_bytes
    f_ = lambda op, B, Nq, Nk, tq, S=0: int(f(op, B, 1, 1, Nq, Nk, tq, 64, S, 32, 128))   # noqa: E731
    big = 2 ** 31 - 1
    assert f_(mala.OP_BWD, 1, 128, 128, big) == 0 and f_(mala.OP_BWD, 65535, 128, 128, big - 384 * 65535 + 1) == 0
    assert f_(mala.OP_BWD, 1, big, 128, 0) == 0 and f_(mala.OP_DECODE, 65535, 65535, 128, 0, 1) == 0
    for tq in (2 ** 30, big - 511):
        rows = -(-(tq + 384) // 128) * 128
        assert rows * 64 * 4 <= f_(mala.OP_BWD, 1, 128, 128, tq) <= rows * (64 + 3) * 4 + 10 ** 6
    a, b = f_(mala.OP_BWD, 1, 128, big, 0), f_(mala.OP_BWD, 1, 128, 2 ** 30, 0)
    assert a - b == (2 ** 24 - 2 ** 23) * 16 * 32 * 4
