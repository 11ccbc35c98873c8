"""What lies around the tensors of the state-space block's operators stays out of their results: padding beside the
rows and a workspace that hold NaN give the bits that zeros give.  Tensors of another GPU are refused."""
import math

import pytest
import torch

import paper_1810_09958_amd as isam

pytestmark = pytest.mark.gpu

CODE = {torch.float32: isam.ISAM_F32, torch.bfloat16: isam.ISAM_BF16}
DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
PLACES = pytest.mark.parametrize("off,pad", [(0, 8), (8, 24), (2, 6), (3, 7)])
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


def source(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *shape: torch.randn(shape, generator=g, device="cuda")


@DTYPES
@PLACES
@pytest.mark.parametrize("M,K,N", [(1, 72, 40), (16, 100, 41), (17, 72, 40), (130, 7, 9), (70, 200, 130), (500, 511, 77), (1024, 72, 2048),
                                   (2047, 63, 2111)])
@pytest.mark.parametrize("act", ["gelu", "none"])
def test_linear(M, K, N, off, pad, act, dtype):
    rnd = source(M + K)
    x, W, r, d, bias = rnd(M, K).to(dtype), (rnd(N, K) / math.sqrt(K)).to(dtype), rnd(M, N).to(dtype), rnd(M, N).to(dtype), rnd(N)

    def call(fill):
        a, w, s, g = (beside(t, off, pad, fill) for t in (x, W, r, d))
        out = isam.linear(a, w, bias=bias, activation=act, residual=s, workspace=room(isam.linear_workspace_size(M, K, N, CODE[dtype], False), fill))
        plain = isam.linear(a, w, bias=bias, activation=act, workspace=room(isam.linear_workspace_size(M, K, N, CODE[dtype], False), fill))
        ws = room(isam.linear_backward_workspace_size(M, K, N, CODE[dtype], False), fill)
        return (out, plain, *isam.linear_backward(a, w, g, bias=bias, activation=act, workspace=ws))

    same(call)


@DTYPES
@PLACES
@pytest.mark.parametrize("T,B,C,K", [(1, 3, 40, 4), (9, 2, 33, 3), (70, 3, 6, 4), (300, 2, 130, 2), (40, 2, 3, 5)])
def test_causal_conv(T, B, C, K, off, pad, dtype):
    rnd = source(T + C)
    x, dy, state, ds = rnd(T, B, C).to(dtype), rnd(T, B, C).to(dtype), rnd(K - 1, B, C).to(dtype), rnd(K - 1, B, C).to(dtype)
    w, opt = rnd(K, C), dict(bias=rnd(C), state=state, reset=rnd(T, B) > 2)

    def call(fill):
        a, d, y, dx = (beside(t, off, pad, fill) for t in (x, dy, torch.zeros_like(x), torch.zeros_like(x)))
        ws = room(isam.causal_conv_backward_workspace_size(T, B, C, K, CODE[dtype]), fill)
        return (*isam.causal_conv(a, w, y=y, **opt), *isam.causal_conv_backward(a, w, d, dstate_T=ds, dx=dx, workspace=ws, **opt))

    same(call)


@DTYPES
@PLACES
@pytest.mark.parametrize("T,B,D,N", [(1, 3, 40, 16), (9, 2, 33, 5), (33, 2, 66, 16), (70, 3, 6, 33), (300, 1, 130, 9), (400, 2, 20, 64)])
def test_selective_scan(T, B, D, N, off, pad, dtype):
    rnd = source(T + D)
    x, dt, z, dy, Bm, Cm = (rnd(T, B, n).to(dtype) for n in (D, D, D, D, N, N))
    A, par = -torch.exp(rnd(D, N)), dict(skip=rnd(D), dt_bias=rnd(D) - 3, reset=rnd(T, B) > 2)
    h0, dh = rnd(B, D, N), rnd(B, D, N)

    def call(fill):
        seq = [beside(x, off, pad, fill), beside(dt, off, pad, fill), A, beside(Bm, off, pad, fill), beside(Cm, off, pad, fill)]
        opt = dict(par, z=beside(z, off, pad, fill))
        states = torch.full(isam.selective_scan_states_shape(T, B, D, N), fill, device="cuda")
        ws = room(isam.selective_scan_workspace_size(T, B, D, N, CODE[dtype]), fill)
        out = isam.selective_scan(*seq, h0=h0, y=beside(torch.zeros_like(x), off, pad, fill), states=states, workspace=ws, **opt)
        ws = room(isam.selective_scan_backward_workspace_size(T, B, D, N, CODE[dtype]), fill)
        grad = isam.selective_scan_backward(*seq, beside(dy, off, pad, fill), states=states, dh_T=dh, workspace=ws,
                                            dx=beside(torch.zeros_like(x), off, pad, fill), dB=beside(torch.zeros_like(Bm), off, pad, fill), **opt)
        return (*out, states, *grad)

    same(call)


@DTYPES
@PLACES
@pytest.mark.parametrize("b,n,V,w", [(1, 1, 5, 3), (2, 4, 255, 4), (3, 2, 4100, 9), (2, 8, 9001, 8)])
def test_beam_step(b, n, V, w, off, pad, dtype):
    rnd = source(V)
    logits, scores = rnd(b, n, V).to(dtype), rnd(b, n)

    def call(fill):
        ws = room(isam.beam_step_workspace_size(b, n, V, w, CODE[dtype]), fill)
        return isam.beam_step(beside(logits, off, pad, fill), scores, width=w, workspace=ws)

    same(call)


def test_tensors_of_another_gpu_are_refused(monkeypatch):
    x, W = torch.zeros((4, 8), device="cuda"), torch.zeros((16, 8), device="cuda")
    seq, A = torch.zeros((4, 1, 8), device="cuda"), torch.zeros((8, 2), device="cuda")
    bc, kept = torch.zeros((4, 1, 2), device="cuda"), torch.zeros((1, 1, 8, 2), device="cuda")
    logits, scores = torch.zeros((1, 2, 9), device="cuda"), torch.zeros((1, 2), device="cuda")
    parent = torch.zeros((1, 2), device="cuda", dtype=torch.int32)
    calls = [lambda: isam.linear(x, W), lambda: isam.linear_backward(x, W, torch.zeros((4, 16), device="cuda")),
             lambda: isam.causal_conv(seq, W[:4]), lambda: isam.causal_conv_backward(seq, W[:4], seq),
             lambda: isam.selective_scan(seq, seq, A, bc, bc), lambda: isam.selective_scan_backward(seq, seq, A, bc, bc, seq, states=kept),
             lambda: isam.beam_step(logits, scores), lambda: isam.beam_reorder(x[:2], parent)]
    for call in calls:
        call()
    torch.cuda.synchronize()
    here = torch.cuda.current_device()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: here + 1)
    monkeypatch.setattr(isam, "lib", lambda: pytest.fail("the library was called"))
    for call in calls:
        with pytest.raises(ValueError):
            call()
