"""C-ABI checks of the recurrent block's entry points that need no GPU: bad arguments are refused
during host-side validation (before any HIP call)."""
import ctypes

import pytest

from paper_1810_09958_amd import _lib

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F32, BF16 = 0, 1


def at(i):
    """Addresses 1 TiB apart (never dereferenced: validation fails before any launch)."""
    return ctypes.c_void_p((i + 1) << 40)


@pytest.fixture(scope="module")
def L():
    return _lib.lib()


def lgru(L, T=8, B=2, H=4, dt=F32, cand=1, gx=at(0), gs=(16, 8), bias=at(1), h0=at(2), reset=at(3), rs=(2, 1), h=at(4),
         hs=(8, 4), hT=at(5), states=at(6), ws=None, wsb=0):
    return L.isam_linear_gru(T, B, H, dt, cand, gx, *gs, bias, h0, reset, *rs, h, *hs, hT, states, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), INVALID), (dict(B=-1), INVALID), (dict(H=-1), INVALID), (dict(dt=2), INVALID), (dict(cand=2), INVALID),
    (dict(gx=None), INVALID), (dict(h=None, hT=None, states=None), INVALID), (dict(gs=(-16, 8)), INVALID),
    (dict(rs=(2, -1)), INVALID), (dict(hs=(7, 4)), INVALID), (dict(hs=(0, 4)), INVALID), (dict(h=at(0)), INVALID),
    (dict(hT=at(2)), INVALID), (dict(states=at(5)), INVALID),
    (dict(T=1 << 40), UNSUPPORTED), (dict(T=1 << 30, B=1 << 10, H=1 << 10), UNSUPPORTED), (dict(gs=(1 << 44, 8)), UNSUPPORTED),
    (dict(T=4096, B=1, gs=(16, 8)), WORKSPACE), (dict(T=4096, B=1, ws=at(7), wsb=64), WORKSPACE),
])
def test_linear_gru_refusals(L, kw, code):
    assert lgru(L, **kw) == code
    assert L.isam_last_error() != b""


def test_linear_gru_no_op(L):
    for kw in (dict(B=0), dict(H=0), dict(B=0, gx=None, h=None, hT=None, states=None)):
        assert lgru(L, **kw) == OK


def lgru_bwd(L, T=8, B=2, H=4, dt=F32, cand=1, gx=at(0), gs=(16, 8), bias=at(1), reset=at(3), rs=(2, 1), states=at(6),
             dh=at(4), ds=(8, 4), dhT=at(5), dg=at(7), dgs=(16, 8), dh0=at(8), db=at(9), ws=at(10), wsb=1 << 20):
    return L.isam_linear_gru_backward(T, B, H, dt, cand, gx, *gs, bias, reset, *rs, states, dh, *ds, dhT, dg, *dgs, dh0, db,
                                      ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=-1), INVALID), (dict(dt=-1), INVALID), (dict(cand=-1), INVALID), (dict(states=None), INVALID),
    (dict(dg=None), INVALID), (dict(dgs=(16, 7)), INVALID), (dict(dg=at(0)), INVALID), (dict(dh0=at(5)), INVALID),
    (dict(db=at(1)), INVALID), (dict(ws=at(7)), INVALID), (dict(ds=(-1, 4)), INVALID),
    (dict(ws=None), WORKSPACE), (dict(wsb=100), WORKSPACE), (dict(H=1 << 31), UNSUPPORTED),
])
def test_linear_gru_backward_refusals(L, kw, code):
    assert lgru_bwd(L, **kw) == code
    assert L.isam_last_error() != b""


def test_linear_gru_workspace(L):
    # one tile of time: nothing; more hand the state on through the workspace
    assert L.isam_linear_gru_workspace_size(64, 64, 1024, BF16) == 0
    assert L.isam_linear_gru_workspace_size(256, 64, 1024, BF16) == 0
    assert L.isam_linear_gru_workspace_size(257, 1, 64, BF16) >= 2 * 64 * 12
    # the bias gradient's partial sums: a row for each tile of time and sequence
    assert L.isam_linear_gru_backward_workspace_size(64, 3, 100, F32) >= 3 * 200 * 4
    for bad in ((0, 1, 1, F32), (5, 0, 1, F32), (5, 1, -1, F32), (5, 1, 1, 9), (1 << 41, 1, 1, F32)):
        assert L.isam_linear_gru_workspace_size(*bad) == 0
        if bad[0]:
            assert L.isam_linear_gru_backward_workspace_size(*bad) == 0


def norm(L, R=6, D=8, G=1, dt=F32, x=at(0), ldx=8, r=at(1), ldr=8, gate=at(2), wa=at(3), wb=at(4), scale=1.0, eps=1e-6, ro=at(5),
         ldro=8, y=at(6), ldy=8):
    return L.isam_norm_residual(R, D, G, dt, x, ldx, r, ldr, gate, wa, wb, scale, eps, ro, ldro, y, ldy, None)


@pytest.mark.parametrize("kw,code", [
    (dict(R=-1), INVALID), (dict(D=-1), INVALID), (dict(dt=2), INVALID), (dict(G=4), INVALID), (dict(G=0), INVALID),
    (dict(G=-1), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(r=None), INVALID), (dict(wb=None), INVALID), (dict(y=None), INVALID), (dict(ro=None), INVALID),
    (dict(x=None), INVALID), (dict(x=None, ro=None, gate=None), INVALID), (dict(ldx=7), INVALID), (dict(ldy=7), INVALID),
    (dict(y=at(0)), INVALID), (dict(y=at(1)), INVALID), (dict(ro=at(0)), INVALID), (dict(ro=at(1), ldro=9), INVALID),
    (dict(ro=at(1), y=at(1)), INVALID), (dict(D=16385, ldx=20000, ldr=20000, ldro=20000, ldy=20000), UNSUPPORTED),
])
def test_norm_residual_refusals(L, kw, code):
    assert norm(L, **kw) == code
    assert L.isam_last_error() != b""


def norm_bwd(L, R=6, D=8, G=1, dt=F32, x=at(0), r=at(1), gate=at(2), wa=at(3), wb=at(4), dy=at(5), dro=at(6), lddro=8, dx=at(7),
             dr=at(8), dg=at(9), da=at(10), db=at(11), ws=at(12), wsb=1 << 20):
    return L.isam_norm_residual_backward(R, D, G, dt, x, 8, r, 8, gate, wa, wb, 1.0, 1e-6, dy, 8, dro, lddro, dx, 8, dr, 8, dg, da,
                                         db, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(R=-1), INVALID), (dict(G=5), INVALID), (dict(dy=None), INVALID), (dict(dr=None), INVALID), (dict(dx=None), INVALID),
    (dict(x=None), INVALID), (dict(gate=None), INVALID), (dict(wa=None), INVALID), (dict(dx=at(0)), INVALID),
    (dict(dr=at(6), lddro=9), INVALID), (dict(dg=at(2)), INVALID), (dict(da=at(11)), INVALID), (dict(ws=at(7)), INVALID),
    (dict(ws=None), WORKSPACE), (dict(wsb=100), WORKSPACE),
])
def test_norm_residual_backward_refusals(L, kw, code):
    assert norm_bwd(L, **kw) == code
    assert L.isam_last_error() != b""


def test_norm_residual_no_op_and_workspace(L):
    assert norm(L, R=0) == OK and norm(L, D=0) == OK
    assert L.isam_norm_residual_backward_workspace_size(100, 64, 1, BF16) >= 3 * 64 * 4
    for bad in ((0, 64, 1, F32), (4, 0, 1, F32), (4, 16385, 1, F32), (4, 64, 1, 7)):
        assert L.isam_norm_residual_backward_workspace_size(*bad) == 0


def gffn(L, M=40, K=16, F=8, dt=BF16, act=1, x=at(0), ldx=16, W=at(1), ldw=16, bias=at(2), out=at(3), ldo=8, ws=None, wsb=0):
    return L.isam_gated_ffn(M, K, F, dt, act, x, ldx, W, ldw, bias, out, ldo, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(M=-1), INVALID), (dict(K=0), INVALID), (dict(F=-1), INVALID), (dict(dt=3), INVALID), (dict(act=3), INVALID),
    (dict(act=-1), INVALID), (dict(x=None), INVALID), (dict(W=None), INVALID), (dict(out=None), INVALID), (dict(ldx=15), INVALID),
    (dict(ldw=15), INVALID), (dict(ldo=7), INVALID), (dict(out=at(0)), INVALID), (dict(out=at(2)), INVALID),
    (dict(dt=F32, K=1600, ldx=1600, ldw=1600), WORKSPACE), (dict(ldx=17), WORKSPACE), (dict(K=15), WORKSPACE), (dict(ldx=17, ws=at(5), wsb=64), WORKSPACE),
    (dict(ldx=17, ws=at(3), wsb=1 << 20), INVALID),
    (dict(M=1 << 20, ldx=1 << 11), UNSUPPORTED), (dict(M=1 << 20, F=1 << 12, ldo=1 << 12), UNSUPPORTED),
    (dict(F=1 << 20, ldw=1 << 12), UNSUPPORTED),
])
def test_gated_ffn_refusals(L, kw, code):
    assert gffn(L, **kw) == code
    assert L.isam_last_error() != b""


def test_gated_ffn_fp32_workspace(L):
    size = L.isam_gated_ffn_workspace_size
    assert size(40, 16, 8, F32, 0) == 0 and size(500, 511, 771, F32, 0) == 0     # few tiles: the block's own kernel
    assert size(2000, 130, 1501, F32, 1) >= 2000 * 2 * 1501 * 4                  # beyond: both projections in memory
    # the gradient's rows of [dg du] end on 16 bytes
    assert L.isam_gated_ffn_backward_workspace_size(40, 16, 9, F32, 1) >= 40 * 24 * 4


def gffn_bwd(L, M=40, K=16, F=8, dt=BF16, act=1, x=at(0), ldx=16, W=at(1), bias=at(2), do=at(3), lddo=8, dx=at(4), dW=at(5), db=at(6),
             ws=at(7), wsb=1 << 24):
    return L.isam_gated_ffn_backward(M, K, F, dt, act, x, ldx, W, 16, bias, do, lddo, dx, 16, dW, 16, db, ws, wsb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(M=-1), INVALID), (dict(act=5), INVALID), (dict(do=None), INVALID), (dict(dx=None, dW=None, db=None), INVALID),
    (dict(lddo=7), INVALID), (dict(dx=at(0)), INVALID), (dict(dW=at(1)), INVALID), (dict(db=at(2)), INVALID),
    (dict(ws=at(5)), INVALID), (dict(ws=None), WORKSPACE), (dict(wsb=10), WORKSPACE), (dict(F=0), INVALID),
])
def test_gated_ffn_backward_refusals(L, kw, code):
    assert gffn_bwd(L, **kw) == code
    assert L.isam_last_error() != b""


def test_gated_ffn_workspace(L):
    assert gffn(L, M=0) == OK and gffn(L, F=0) == OK
    q = L.isam_gated_ffn_workspace_size
    assert q(4096, 1024, 4096, BF16, 1) == 0 and q(16, 33, 17, F32, 0) == 0
    assert q(4096, 1024, 4096, BF16, 0) == 2 * 1024 * (4096 + 8192) + 255          # both copied
    assert q(100, 33, 64, BF16, 1) == 2 * (100 * 40 + 128 * 40) + 255 + (-(2 * 100 * 40)) % 256
    assert q(1000, 1000, 640, F32, 1) >= 1000 * 1280 * 4
    for bad in ((0, 8, 8, F32, 1), (8, 0, 8, F32, 1), (8, 8, 0, BF16, 1), (8, 8, 8, 5, 1)):
        assert q(*bad) == 0 and L.isam_gated_ffn_backward_workspace_size(*bad) == 0
