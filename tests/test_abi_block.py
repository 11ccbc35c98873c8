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
    # enough sequences and channels: one segment, nothing but the bias gradient's partial sums
    assert L.isam_linear_gru_workspace_size(4096, 64, 1024, BF16) == 0
    assert L.isam_linear_gru_backward_workspace_size(4096, 64, 1024, BF16) == 64 * 2048 * 4 + 255
    # few: two numbers per segment and channel besides
    assert L.isam_linear_gru_workspace_size(32768, 1, 64, BF16) > 0
    for bad in ((0, 1, 1, F32), (5, 0, 1, F32), (5, 1, -1, F32), (5, 1, 1, 9), (1 << 41, 1, 1, F32)):
        assert L.isam_linear_gru_workspace_size(*bad) == 0
        if bad[0]:
            assert L.isam_linear_gru_backward_workspace_size(*bad) == 0
