"""What lies around an operator's tensors stays out of its results: padding beside the rows and a
workspace that hold NaN give the bits that zeros give."""
import math

import pytest
import torch

import paper_1810_09958_amd as isam

pytestmark = pytest.mark.gpu

CODE = {torch.float32: isam.ISAM_F32, torch.bfloat16: isam.ISAM_BF16}
NAN = float("nan")


def beside(t, off, pad, fill):
    """t inside wider rows (last dimension) whose other values are `fill`."""
    w = torch.full((*t.shape[:-1], t.shape[-1] + pad), fill, device="cuda", dtype=t.dtype)
    w[..., off:off + t.shape[-1]] = t
    return w[..., off:off + t.shape[-1]]


def room(nbytes, fill):
    return torch.full((max(nbytes, 1),), 0xFF if fill != fill else 0, device="cuda", dtype=torch.uint8)


def same(call):
    good, bad = call(0.0), call(NAN)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(good, bad)):
        assert (a is None) == (b is None)
        if a is not None:
            assert torch.isfinite(a.float()).all(), i
            assert torch.equal(a, b), i


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off,pad", [(0, 8), (8, 24), (3, 7)])
@pytest.mark.parametrize("M,K,F", [(1, 72, 40), (16, 100, 41), (17, 72, 40), (130, 7, 9), (70, 200, 65), (500, 511, 77), (600, 700, 900),
                                   (1024, 72, 2048), (1025, 130, 2111), (2048, 72, 4096), (2047, 63, 4095)])
def test_gated_ffn(M, K, F, off, pad, dtype):
    g = torch.Generator(device="cuda").manual_seed(M + K)

    def rnd(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    x, W, do = rnd(M, K).to(dtype), (rnd(2 * F, K) / math.sqrt(K)).to(dtype), rnd(M, F).to(dtype)
    bias = rnd(2 * F)

    def call(fill):
        a, w, d = beside(x, off, pad, fill), beside(W, off, pad, fill), beside(do, off, pad, fill)
        ws = room(isam.gated_ffn_workspace_size(M, K, F, CODE[dtype], False), fill)
        out = isam.gated_ffn(a, w, bias=bias, workspace=ws)
        ws = room(isam.gated_ffn_backward_workspace_size(M, K, F, CODE[dtype], False), fill)
        return (out, *isam.gated_ffn_backward(a, w, d, bias=bias, workspace=ws))

    same(call)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off,pad", [(0, 8), (8, 24), (3, 7)])
@pytest.mark.parametrize("R,D,G", [(1, 1, 1), (9, 200, 3), (40, 203, 40), (3000, 72, 10), (300, 1030, 1), (2600, 600, 1300), (33, 5000, 11),
                                   (20, 16384, 1)])
def test_norm_residual(R, D, G, off, pad, dtype):
    g = torch.Generator(device="cuda").manual_seed(R + D)

    def rnd(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    x, r, dy, dr = (rnd(R, D).to(dtype) for _ in range(4))
    opt = dict(w_pre=rnd(D), w_post=rnd(D), gate=rnd(G, D).to(dtype))

    def call(fill):
        xs, rs, ys, ds = (beside(t, off, pad, fill) for t in (x, r, dy, dr))
        ws = room(isam.norm_residual_backward_workspace_size(R, D, G, CODE[dtype]), fill)
        return (*isam.norm_residual(xs, rs, **opt), *isam.norm_residual_backward(xs, rs, ys, dr_out=ds, workspace=ws, **opt))

    same(call)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off,pad", [(0, 8), (2, 6), (3, 7)])
@pytest.mark.parametrize("T,B,H", [(1, 3, 40), (9, 2, 33), (64, 2, 66), (129, 2, 6), (300, 3, 37), (700, 2, 130), (3000, 1, 2)])
def test_linear_gru(T, B, H, off, pad, dtype):
    g = torch.Generator(device="cuda").manual_seed(T + H)

    def rnd(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    gx, dh = rnd(T, B, 2 * H).to(dtype), rnd(T, B, H).to(dtype)
    opt = dict(bias=rnd(2 * H), reset=torch.rand((T, B), generator=g, device="cuda") < 0.02)
    h0, dh_T = rnd(B, H), rnd(B, H)

    def call(fill):
        a, d = beside(gx, off, pad, fill), beside(dh, off, pad, fill)
        hs, dg = beside(torch.zeros_like(dh), off, pad, fill), beside(torch.zeros_like(gx), off, pad, fill)
        states = torch.full(isam.linear_gru_states_shape(T, B, H), fill, device="cuda")
        ws = room(isam.linear_gru_workspace_size(T, B, H, CODE[dtype]), fill)
        h, h_T = isam.linear_gru(a, h0=h0, h_seq=hs, states=states, workspace=ws, **opt)
        ws = room(isam.linear_gru_backward_workspace_size(T, B, H, CODE[dtype]), fill)
        return (h, h_T, states, *isam.linear_gru_backward(a, d, states=states, dh_T=dh_T, dgx=dg, workspace=ws, **opt))

    same(call)
