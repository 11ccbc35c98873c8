"""C-ABI checks of the state-space block's and beam search's entry points that need no GPU: bad arguments are
refused during host-side validation (before any HIP call)."""
import ctypes
import random

import pytest

from paper_1810_09958_amd import _lib

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16 = 0, 1
NONE = 3


def at(i, off=0):
    """Addresses 1 TiB apart (never dereferenced: validation fails before any launch)."""
    return ctypes.c_void_p(((i + 1) << 40) + off)


@pytest.fixture(scope="module")
def L():
    return _lib.lib()


def refused(L, code, got):
    assert got == code
    assert L.isam_last_error() != b""


def scan(L, T=9, B=2, D=4, N=3, dt=F32, x=(at(0), 8, 4), d=(at(1), 8, 4), A=at(2), Bm=(at(3), 6, 3), Cm=(at(4), 6, 3), skip=at(5),
         z=(at(6), 8, 4), bias=at(7), h0=at(8), reset=(at(9), 2, 1), y=(at(10), 8, 4), hT=at(11), states=at(12), ws=at(13), wsb=1 << 24):
    return L.isam_selective_scan(T, B, D, N, dt, *x, *d, A, *Bm, *Cm, skip, *z, bias, h0, *reset, *y, hT, states, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), INVALID), (dict(B=-1), INVALID), (dict(D=-1), INVALID), (dict(N=0), INVALID), (dict(N=-1), INVALID), (dict(dt=2), INVALID),
    (dict(N=65), UNSUPPORTED), (dict(T=1 << 40), UNSUPPORTED), (dict(T=1 << 30, B=1 << 10, D=1 << 10), UNSUPPORTED),
    (dict(x=(None, 8, 4)), INVALID), (dict(d=(None, 8, 4)), INVALID), (dict(A=None), INVALID), (dict(Bm=(None, 6, 3)), INVALID),
    (dict(Cm=(None, 6, 3)), INVALID), (dict(y=(None, 0, 0), hT=None, states=None), INVALID),
    (dict(x=(at(0), -8, 4)), INVALID), (dict(z=(at(6), 8, -4)), INVALID), (dict(reset=(at(9), -1, 1)), INVALID),
    (dict(y=(at(10), 7, 4)), INVALID), (dict(y=(at(10), 0, 4)), INVALID), (dict(y=(at(0), 8, 4)), INVALID),
    (dict(y=(at(0, 12), 8, 4)), INVALID), (dict(y=(at(6), 8, 4)), INVALID), (dict(hT=at(8)), INVALID), (dict(hT=at(2)), INVALID),
    (dict(states=at(11)), INVALID), (dict(hT=at(10)), INVALID), (dict(y=(at(9), 8, 4)), INVALID), (dict(hT=at(9)), INVALID),
    (dict(x=(at(0), 1 << 44, 4)), UNSUPPORTED), (dict(x=(at(0), 1 << 27, 4)), UNSUPPORTED), (dict(reset=(at(9), 1 << 27, 1)), UNSUPPORTED),
    (dict(T=4096, B=1, ws=None, wsb=0), WORKSPACE), (dict(T=4096, B=1, wsb=64), WORKSPACE), (dict(T=4096, B=1, ws=at(0)), INVALID),
])
def test_selective_scan_refusals(L, kw, code):
    refused(L, code, scan(L, **kw))


def test_selective_scan_no_op_and_workspace(L):
    for kw in (dict(B=0), dict(D=0), dict(B=0, x=(None, 0, 0), y=(None, 0, 0), hT=None, states=None)):
        assert scan(L, **kw) == OK
    q, qb = L.isam_selective_scan_workspace_size, L.isam_selective_scan_backward_workspace_size
    assert q(8, 64, 1024, 16, BF16) == 0 and q(4096, 64, 4096, 16, BF16) == 0       # few tokens; channels that fill the chip
    assert q(4096, 1, 64, 16, BF16) >= 2 * 64 * 17 * 4
    assert qb(40, 2, 100, 16, F32) >= 40 * 2 * 32 * 4 + 2 * 100 * 18 * 4
    for bad in ((0, 1, 1, 1, F32), (5, 0, 1, 1, F32), (5, 1, 0, 1, F32), (5, 1, 1, 0, F32), (5, 1, 1, 65, F32), (5, 1, 1, 1, 9), (1 << 41, 1, 1, 1, F32)):
        assert q(*bad) == 0 and qb(*bad) == 0


def test_rows_of_one_tensor(L):
    # An output among the rows of an input with the same strides: refused where an element is shared, else not.  (The marks'
    # stride is refused by a later check, so that no call is launched.)
    far = (at(9), 1 << 27, 1)
    T, B, D, g = 9, 3, 4, random.Random(1)
    refused(L, UNSUPPORTED, scan(L, T=T, B=B, x=(at(0), 24, 4), y=(at(0, 48), 24, 4), reset=far))        # [T][2][B][D]
    refused(L, UNSUPPORTED, scan(L, T=T, B=B, x=(at(0), 12, 4), y=(at(0, 9 * 48), 12, 4), reset=far))    # [2][T][B][D]
    met = 0
    for _ in range(600):
        if g.random() < 0.5:
            sb = g.randint(D, 14)
            st = g.randint((B - 1) * sb + D, 70)
        else:
            st = g.randint(D, 14)
            sb = g.randint((T - 1) * st + D, 200)
        gap = g.randint(-80, 80) * g.choice((1, 1, 4))
        rows = {t * st + b * sb + c for t in range(T) for b in range(B) for c in range(D)}
        shared = any(gap + v in rows for v in rows)
        met += shared
        code = scan(L, T=T, B=B, x=(at(0, 1 << 20), st, sb), y=(at(0, (1 << 20) + 4 * gap), st, sb), reset=far)
        refused(L, INVALID if shared else UNSUPPORTED, code)
        shared = any(gap + v in rows for t in range(T) for b in range(B) for v in range(t * st + b * sb, t * st + b * sb + 3))
        code = scan(L, T=T, B=B, y=(at(0, 1 << 20), st, sb), Bm=(at(0, (1 << 20) + 4 * gap), st, sb), reset=far)       # (rows of 3)
        refused(L, INVALID if shared else UNSUPPORTED, code)
    assert 200 < met < 500


def scan_bwd(L, T=9, B=2, D=4, N=3, dt=F32, x=(at(0), 8, 4), d=(at(1), 8, 4), A=at(2), Bm=(at(3), 6, 3), Cm=(at(4), 6, 3), skip=at(5),
             z=(at(6), 8, 4), bias=at(7), reset=(at(9), 2, 1), states=at(12), dy=(at(10), 8, 4), dhT=at(11), dx=(at(14), 8, 4),
             dd=(at(15), 8, 4), dA=at(16), dB=(at(17), 6, 3), dC=(at(18), 6, 3), dskip=at(19), dz=(at(20), 8, 4), dbias=at(21), dh0=at(22),
             ws=at(13), wsb=1 << 24):
    return L.isam_selective_scan_backward(T, B, D, N, dt, *x, *d, A, *Bm, *Cm, skip, *z, bias, *reset, states, *dy, dhT, *dx, *dd, dA, *dB,
                                          *dC, dskip, *dz, dbias, dh0, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), INVALID), (dict(dt=-1), INVALID), (dict(N=65), UNSUPPORTED), (dict(states=None), INVALID), (dict(dx=(None, 0, 0)), INVALID),
    (dict(dd=(None, 0, 0)), INVALID), (dict(dB=(None, 0, 0)), INVALID), (dict(dC=(None, 0, 0)), INVALID), (dict(z=(None, 0, 0)), INVALID),
    (dict(dx=(at(14), 8, 3)), INVALID), (dict(dx=(at(0), 8, 4)), INVALID), (dict(dd=(at(14), 8, 4)), INVALID), (dict(dB=(at(18), 6, 3)), INVALID),
    (dict(dB=(at(18, 4), 6, 3)), INVALID), (dict(dA=at(2)), INVALID), (dict(dskip=at(5)), INVALID), (dict(dh0=at(11)), INVALID),
    (dict(dh0=at(12)), INVALID), (dict(dx=(at(9), 8, 4)), INVALID), (dict(ws=at(14)), INVALID), (dict(dy=(at(10), -1, 4)), INVALID),
    (dict(ws=None), WORKSPACE), (dict(wsb=64), WORKSPACE), (dict(dx=(at(14), 1 << 27, 4)), UNSUPPORTED),
])
def test_selective_scan_backward_refusals(L, kw, code):
    refused(L, code, scan_bwd(L, **kw))


def test_selective_scan_backward_without_channels(L):
    none = dict(D=0, x=(None, 0, 0), d=(None, 0, 0), A=None, z=(None, 0, 0), ws=None, wsb=0)
    assert scan_bwd(L, T=0, **none) == OK and scan_bwd(L, B=0, **none) == OK
    for kw in (dict(dB=(None, 0, 0)), dict(dC=(None, 0, 0)), dict(dB=(at(18), 6, 3)), dict(dC=(at(18), 5, 3)), dict(dB=(at(17), -6, 3))):
        refused(L, INVALID, scan_bwd(L, **none, **kw))


def conv(L, T=9, B=2, C=8, K=4, dt=BF16, act=1, x=(at(0), 16, 8), w=at(1), bias=at(2), state=at(3), reset=(at(4), 2, 1), y=(at(5), 16, 8),
         sT=at(6)):
    return L.isam_causal_conv(T, B, C, K, dt, act, *x, w, bias, state, *reset, *y, sT, None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), INVALID), (dict(B=-1), INVALID), (dict(C=-1), INVALID), (dict(K=0), INVALID), (dict(dt=3), INVALID), (dict(act=2), INVALID),
    (dict(act=0), INVALID), (dict(K=7), UNSUPPORTED), (dict(T=1 << 41), UNSUPPORTED), (dict(x=(None, 16, 8)), INVALID), (dict(w=None), INVALID),
    (dict(y=(None, 0, 0), sT=None), INVALID), (dict(x=(at(0), -1, 8)), INVALID), (dict(y=(at(5), 15, 8)), INVALID), (dict(y=(at(0), 16, 8)), INVALID),
    (dict(sT=at(3)), INVALID), (dict(sT=at(5)), INVALID), (dict(sT=at(1)), INVALID), (dict(y=(at(4), 16, 8)), INVALID),
    (dict(reset=(at(4), 1, -1)), INVALID), (dict(x=(at(0), 1 << 44, 8)), UNSUPPORTED),
])
def test_causal_conv_refusals(L, kw, code):
    refused(L, code, conv(L, **kw))


def conv_bwd(L, T=9, B=2, C=8, K=4, dt=BF16, act=1, x=(at(0), 16, 8), w=at(1), bias=at(2), state=at(3), reset=(at(4), 2, 1), dy=(at(5), 16, 8),
             dsT=at(6), dx=(at(7), 16, 8), ds=at(8), dw=at(9), db=at(10), ws=at(11), wsb=1 << 20):
    return L.isam_causal_conv_backward(T, B, C, K, dt, act, *x, w, bias, state, *reset, *dy, dsT, *dx, ds, dw, db, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), INVALID), (dict(act=5), INVALID), (dict(K=7), UNSUPPORTED), (dict(x=(None, 0, 0)), INVALID), (dict(w=None), INVALID),
    (dict(dx=(None, 0, 0), ds=None, dw=None, db=None), INVALID), (dict(dx=(at(7), 16, 7)), INVALID), (dict(dx=(at(0), 16, 8)), INVALID),
    (dict(ds=at(6)), INVALID), (dict(dw=at(1)), INVALID), (dict(db=at(9)), INVALID), (dict(ws=at(7)), INVALID), (dict(ws=None), WORKSPACE),
    (dict(wsb=64), WORKSPACE),
])
def test_causal_conv_backward_refusals(L, kw, code):
    refused(L, code, conv_bwd(L, **kw))


@pytest.mark.parametrize("C,dt,fits", [((1 << 30) + 1, F32, False), (1 << 30, F32, True), ((1 << 31) - 1, F32, False), ((1 << 31) - 1, BF16, True)])
def test_causal_conv_rows_of_32_bits(L, C, dt, fits):
    # a lane's place in its row: rows of more than 2^32 bytes are refused, in the query too
    assert (L.isam_causal_conv_backward_workspace_size(1, 1, C, 4, dt) > 0) == fits
    kw = dict(T=1, B=1, C=C, dt=dt, x=(at(0), C, C), dx=(at(7), C, C), dy=(at(5), C, C), ws=None)
    refused(L, WORKSPACE if fits else UNSUPPORTED, conv_bwd(L, **kw))
    if not fits:
        refused(L, UNSUPPORTED, conv(L, T=1, B=1, C=C, dt=dt, x=(at(0), C, C), y=(at(5), C, C)))


def test_causal_conv_no_op_and_workspace(L):
    assert conv(L, B=0) == OK and conv(L, C=0) == OK
    q = L.isam_causal_conv_backward_workspace_size
    assert q(9, 2, 8, 4, BF16) >= 2 * 5 * 8 * 4
    for bad in ((0, 2, 8, 4, BF16), (9, 0, 8, 4, BF16), (9, 2, 0, 4, BF16), (9, 2, 8, 0, BF16), (9, 2, 8, 7, BF16), (9, 2, 8, 4, 7)):
        assert q(*bad) == 0


def linear(L, M=40, K=16, N=8, dt=BF16, act=1, x=at(0), ldx=16, W=at(1), ldw=16, bias=at(2), r=at(3), ldr=8, out=at(4), ldo=8, ws=None, wsb=0):
    return L.isam_linear(M, K, N, dt, act, x, ldx, W, ldw, bias, r, ldr, out, ldo, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(M=-1), INVALID), (dict(K=0), INVALID), (dict(N=-1), INVALID), (dict(dt=3), INVALID), (dict(act=4), INVALID), (dict(act=-1), INVALID),
    (dict(x=None), INVALID), (dict(W=None), INVALID), (dict(out=None), INVALID), (dict(ldx=15), INVALID), (dict(ldw=15), INVALID),
    (dict(ldo=7), INVALID), (dict(ldr=7), INVALID), (dict(out=at(0)), INVALID), (dict(out=at(2)), INVALID), (dict(out=at(3), ldo=9), INVALID),
    (dict(out=at(3, 2)), INVALID), (dict(M=100, ldx=17), WORKSPACE), (dict(M=100, K=15), WORKSPACE), (dict(dt=F32, M=4000, K=2000, N=4000, ldx=2000, ldw=2000, ldr=4000, ldo=4000), WORKSPACE),
    (dict(M=100, ldx=17, ws=at(5), wsb=64), WORKSPACE), (dict(M=100, ldx=17, ws=at(4), wsb=1 << 20), INVALID),
    (dict(M=1 << 20, ldx=1 << 11), UNSUPPORTED), (dict(M=1 << 20, N=1 << 12, ldo=1 << 12, ldr=1 << 12), UNSUPPORTED),
    (dict(N=1 << 20, ldw=1 << 12, ldr=1 << 20, ldo=1 << 20), UNSUPPORTED),
])
def test_linear_refusals(L, kw, code):
    refused(L, code, linear(L, **kw))


def linear_bwd(L, M=40, K=16, N=8, dt=BF16, act=1, x=at(0), ldx=16, W=at(1), bias=at(2), do=at(3), lddo=8, dx=at(4), dW=at(5), db=at(6),
               ws=at(7), wsb=1 << 24):
    return L.isam_linear_backward(M, K, N, dt, act, x, ldx, W, 16, bias, do, lddo, dx, 16, dW, 16, db, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(M=-1), INVALID), (dict(act=5), INVALID), (dict(do=None), INVALID), (dict(dx=None, dW=None, db=None), INVALID), (dict(lddo=7), INVALID),
    (dict(dx=at(0)), INVALID), (dict(dW=at(1)), INVALID), (dict(db=at(2)), INVALID), (dict(ws=at(5)), INVALID), (dict(ws=None), WORKSPACE),
    (dict(wsb=10), WORKSPACE), (dict(N=0), INVALID), (dict(act=NONE, ws=None), WORKSPACE),
])
def test_linear_backward_refusals(L, kw, code):
    refused(L, code, linear_bwd(L, **kw))


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("act", [0, 1, 2, NONE])
@pytest.mark.parametrize("K,N", [(16, 8), (15, 7), (300, 300), (512, 512), (4096, 1024)])
def test_linear_backward_of_no_rows(L, K, N, act, dt):
    # the plan of an empty batch needs no workspace, as its query says; dx has no values, so nothing is launched
    assert L.isam_linear_backward_workspace_size(0, K, N, dt, 1) == 0
    assert L.isam_linear_backward(0, K, N, dt, act, at(0), K, at(1), K, at(2), at(3), N, at(4), K, None, K, None, None, 0, None) == OK


def test_linear_no_op_and_workspace(L):
    assert linear(L, M=0) == OK and linear(L, N=0) == OK
    q, qb = L.isam_linear_workspace_size, L.isam_linear_backward_workspace_size
    assert q(16, 33, 17, F32, 0) == 0 and q(40, 16, 8, F32, 0) == 0            # few rows; few tiles
    assert q(4096, 1024, 4096, BF16, 0) >= 2 * 1024 * (4096 + 4096)            # both copied
    assert q(2000, 4000, 3001, F32, 1) >= 2000 * 3001 * 4                      # the product in memory
    for bad in ((0, 8, 8, F32, 1), (8, 0, 8, F32, 1), (8, 8, 0, BF16, 1), (8, 8, 8, 5, 1)):
        assert q(*bad) == 0 and qb(*bad) == 0


def beam(L, b=2, n=3, V=50, w=4, dt=F32, lg=(at(0), 150, 50), sc=at(1), fin=at(2), end=2, so=at(3), pa=at(4), to=at(5), fo=at(6), ws=at(7),
         wsb=1 << 20):
    return L.isam_beam_step(b, n, V, w, dt, *lg, sc, fin, end, so, pa, to, fo, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(b=-1), INVALID), (dict(n=0), INVALID), (dict(V=0), INVALID), (dict(w=0), INVALID), (dict(w=151), UNSUPPORTED), (dict(w=16, V=5), INVALID),
    (dict(n=65), UNSUPPORTED), (dict(w=65), UNSUPPORTED), (dict(V=1 << 30), UNSUPPORTED), (dict(b=1 << 40), UNSUPPORTED), (dict(dt=2), INVALID),
    (dict(end=50), INVALID), (dict(end=-1), INVALID), (dict(lg=(None, 150, 50)), INVALID), (dict(sc=None), INVALID), (dict(so=None), INVALID),
    (dict(pa=None), INVALID), (dict(to=None), INVALID), (dict(lg=(at(0), -1, 50)), INVALID), (dict(so=at(1)), INVALID), (dict(pa=at(5)), INVALID),
    (dict(fo=at(2)), INVALID), (dict(ws=at(0)), INVALID), (dict(ws=None), WORKSPACE), (dict(wsb=64), WORKSPACE),
    (dict(lg=(at(0), 1 << 50, 50)), UNSUPPORTED),
])
def test_beam_step_refusals(L, kw, code):
    refused(L, code, beam(L, **kw))


def reorder(L, o=2, b=2, n=3, w=3, row=20, src=at(0), pa=at(1), dst=at(2)):
    return L.isam_beam_reorder(o, b, n, w, row, src, pa, dst, None)


@pytest.mark.parametrize("kw,code", [
    (dict(o=-1), INVALID), (dict(b=-1), INVALID), (dict(n=0), INVALID), (dict(w=0), INVALID), (dict(row=-1), INVALID), (dict(src=None), INVALID),
    (dict(pa=None), INVALID), (dict(dst=None), INVALID), (dict(dst=at(0)), INVALID), (dict(dst=at(0, 230)), INVALID), (dict(dst=at(1)), INVALID),
    (dict(row=1 << 41), UNSUPPORTED), (dict(o=1 << 30, row=1 << 20), UNSUPPORTED),
])
def test_beam_reorder_refusals(L, kw, code):
    refused(L, code, reorder(L, **kw))


def test_beam_no_op_and_workspace(L):
    assert beam(L, b=0) == OK
    for kw in (dict(o=0), dict(b=0), dict(row=0)):
        assert reorder(L, **kw) == OK
    q = L.isam_beam_step_workspace_size
    assert q(2, 3, 9000, 4, BF16) >= 2 * 3 * 3 * (16 + 8 * 4)
    for bad in ((0, 3, 50, 4, F32), (2, 0, 50, 4, F32), (2, 3, 0, 4, F32), (2, 3, 50, 65, F32), (2, 65, 50, 4, F32), (2, 3, 50, 4, 9)):
        assert q(*bad) == 0
