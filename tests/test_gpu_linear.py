"""GPU parity of the projection with its epilogue and of its gradient against the formulas in 64 bits.

Tolerances are error bounds formed beside the 64-bit results, u = 2^-24.  A product over K is good to
(K / 8 + 32) u of its sum of absolute products (sixteen products to an addition; fp32 products are formed to
about 2^-22); the activations and their slopes (at most 1.13 in slope themselves) add 32 u relative, of 1 + |p|;
with an activation dP is rounded to bf16 as operand (up to 2^-8; in two terms up to 16 rows, which lose below
2^-16), sums over M or N as over K; bf16 outputs add another such rounding.  Besides, the relative norm error of
a result of 256 values or more stays below 4e-3 for bf16 (one rounding 1.7e-3, two 2.4e-3) and 2e-6 for fp32."""
import math

import pytest
import torch

import paper_1810_09958_amd as isam

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
NORM = {torch.float32: 2e-6, torch.bfloat16: 4e-3}
ACTS = ("none", "sigmoid", "silu", "gelu")
DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])


def inputs(M, K, N, dtype, seed=0, bias=True, residual=True):
    g = torch.Generator().manual_seed(seed)
    return dict(x=torch.randn((M, K), generator=g).to(dtype).cuda(), W=(torch.randn((N, K), generator=g) / math.sqrt(K)).to(dtype).cuda(),
                bias=(torch.randn(N, generator=g) * 0.3).cuda() if bias else None,
                residual=torch.randn((M, N), generator=g).to(dtype).cuda() if residual else None,
                dout=torch.randn((M, N), generator=g).to(dtype).cuda())


def act(name, p):
    if name == "none":
        return p, torch.ones_like(p)
    if name == "gelu":
        cdf = 0.5 * torch.special.erfc(-p / math.sqrt(2))
        return p * cdf, cdf + p * torch.exp(-p * p / 2) / math.sqrt(2 * math.pi)
    z, w = torch.sigmoid(p), torch.sigmoid(-p)
    return (z, z * w) if name == "sigmoid" else (p * z, z * (1 + p * w))


def mm(a, b):
    return torch.matmul(a.contiguous(), b.contiguous())


def reference(x, name):
    X, W, do = x["x"].double(), x["W"].double(), x["dout"].double()
    (M, K), N = X.shape, W.shape[0]
    b = x["bias"].double() if x["bias"] is not None else torch.zeros(N, device=X.device, dtype=torch.float64)
    r = x["residual"].double() if x["residual"] is not None else torch.zeros_like(do)
    p, ep = mm(X, W.t()) + b, (K / 8 + 32) * U * (mm(X.abs(), W.abs().t()) + b.abs())
    s, ds = act(name, p)
    extra = 0 if name == "none" else 32 * U * (1 + p.abs())
    out = dict(out=(s + r, 1.13 * ep + extra + 2 * U * (s.abs() + r.abs())))
    d = do * ds
    ed = do.abs() * ((0 if name == "none" else ep) + extra) + 2 * U * d.abs()
    out["dbias"] = (d.sum(0), ed.sum(0) + (M / 64 + 64) * U * d.abs().sum(0))
    half = 0 if name == "none" or x["x"].dtype == torch.float32 else 2.0 ** -8 if M > 16 else 2.0 ** -16
    er = ed + half * (d.abs() + ed)
    out["dx"] = (mm(d, W), mm(er + (N / 8 + 32) * U * d.abs(), W.abs()))
    out["dW"] = (mm(d.t(), X), mm((er + (M / 8 + 32) * U * d.abs()).t(), X.abs()))
    return out


def check(got, ref, name):
    val, bound = ref
    bound = bound + HALF[got.dtype] * (val.abs() + bound) + 1e-30
    err = (got.double() - val).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / bound).max()):.2f} bounds"
    norm = float(val.norm())
    assert val.numel() < 256 or float(err.norm()) <= NORM[got.dtype] * norm + 1e-30, f"{name}: norm {float(err.norm()) / norm:.2e}"


def compare(x, name, backward=True):
    ref = reference(x, name)
    check(isam.linear(x["x"], x["W"], bias=x["bias"], activation=name, residual=x["residual"]), ref["out"], "out")
    if x["residual"] is not None:     # in place
        r = x["residual"].clone()
        assert isam.linear(x["x"], x["W"], bias=x["bias"], activation=name, residual=r, out=r) is r
        check(r, ref["out"], "out in place")
    if backward:
        got = dict(zip(("dx", "dW", "dbias"), isam.linear_backward(x["x"], x["W"], x["dout"], bias=x["bias"], activation=name)))
        for k, v in got.items():
            if v is not None:
                check(v, ref[k], k)


@DTYPES
@pytest.mark.parametrize("M,K,N", [(1, 64, 64), (1, 1, 1), (2, 8, 16), (3, 1000, 17), (7, 33, 100), (16, 4096, 48), (16, 72, 515), (17, 64, 64),
                                   (1, 5000, 333), (5, 333, 1001)])
def test_few_rows(M, K, N, dtype):
    for i, name in enumerate(ACTS):
        compare(inputs(M, K, N, dtype, seed=M + i, bias=i != 1, residual=i != 2), name)


@DTYPES
@pytest.mark.parametrize("M,K,N", [(33, 64, 64), (64, 128, 192), (65, 72, 33), (100, 200, 65), (200, 520, 80), (130, 7, 9), (64, 1, 64),
                                   (300, 511, 77), (1000, 96, 1), (40, 3000, 200)])
def test_small_tiles(M, K, N, dtype):
    for i, name in enumerate(ACTS):
        compare(inputs(M, K, N, dtype, seed=M + i, bias=i != 1, residual=i != 3), name)


@DTYPES
@pytest.mark.parametrize("M,K,N", [(600, 200, 2100), (1300, 130, 1500), (2048, 64, 2047), (3000, 100, 2600)])
def test_large_tiles(M, K, N, dtype):
    for i, name in enumerate(("gelu", "none")):
        compare(inputs(M, K, N, dtype, seed=M + i, bias=i == 0), name)


@pytest.mark.parametrize("M,K,N", [(1, 210, 76), (2, 64, 128), (5, 333, 1001), (16, 1000, 31), (16, 72, 515)])
def test_gradient_of_few_rows_rounds_once(M, K, N):
    # dx and dW within one rounding of the output, at most 2^-9 of each value and so of the norm, and what two
    # terms of 8 bits lose, below 2^-13
    for i, name in enumerate(ACTS):
        x = inputs(M, K, N, torch.bfloat16, seed=M + i, bias=i != 1)
        ref = reference(x, name)
        for k, v in zip(("dx", "dW"), isam.linear_backward(x["x"], x["W"], x["dout"], bias=x["bias"], activation=name)):
            val = ref[k][0]
            assert float((v.double() - val).norm()) <= (2.0 ** -9 + 2.0 ** -13) * float(val.norm()), k
