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


@DTYPES
@pytest.mark.parametrize("M,K,N", [(5, 72, 40), (70, 72, 40), (300, 200, 65), (500, 511, 77), (1500, 130, 1100)])
def test_strided_rows(M, K, N, dtype):
    # every matrix as a slice of wider rows, off 16 bytes; nothing beside the rows is touched
    for name in ("gelu", "none"):
        x = inputs(M, K, N, dtype, seed=M)
        ref = reference(x, name)

        def wide(t, off, fill):
            w = torch.full((t.shape[0], t.shape[1] + 11), fill, device="cuda", dtype=t.dtype)
            w[:, off:off + t.shape[1]] = t
            return w, w[:, off:off + t.shape[1]]

        xs, ws, rs, ds = (wide(x[k], o, float("nan"))[1] for k, o in (("x", 3), ("W", 1), ("residual", 5), ("dout", 2)))
        out_w, out = wide(torch.zeros_like(x["dout"]), 3, 7.0)
        dx_w, dx = wide(torch.zeros_like(x["x"]), 1, 7.0)
        dW_w, dW = wide(torch.zeros_like(x["W"]), 4, 7.0)
        isam.linear(xs, ws, bias=x["bias"], activation=name, residual=rs, out=out)
        _, _, db = isam.linear_backward(xs, ws, ds, bias=x["bias"], activation=name, dx=dx, dW=dW)
        for k, v in (("out", out), ("dx", dx), ("dW", dW), ("dbias", db)):
            check(v, ref[k], f"{name} {k}")
        for w, off, n in ((out_w, 3, N), (dx_w, 1, K), (dW_w, 4, K)):
            assert (w[:, :off] == 7).all() and (w[:, off + n:] == 7).all()


@DTYPES
def test_parts_of_the_gradient(dtype):
    x = inputs(100, 64, 72, dtype)
    for name in ("silu", "none"):
        ref = reference(x, name)
        dx, dW, db = isam.linear_backward(x["x"], x["W"], x["dout"], activation=name, return_dW=False)
        assert dW is None and db is None
        check(dx, ref["dx"] if x["bias"] is None else reference({**x, "bias": None}, name)["dx"], "dx")
        dx, dW, db = isam.linear_backward(x["x"], x["W"], x["dout"], bias=x["bias"], activation=name, return_dx=False)
        assert dx is None
        check(dW, ref["dW"], "dW")
        check(db, ref["dbias"], "dbias")


def test_empty():
    for dtype in (torch.float32, torch.bfloat16):
        e = torch.empty((0, 16), device="cuda", dtype=dtype)
        W = torch.ones((8, 16), device="cuda", dtype=dtype)
        assert isam.linear(e, W).shape == (0, 8)
        dx, dW, db = isam.linear_backward(e, W, torch.empty((0, 8), device="cuda", dtype=dtype), bias=torch.ones(8, device="cuda"))
        assert dx.shape == (0, 16) and (dW == 0).all() and (db == 0).all()
        x, none = torch.ones((5, 16), device="cuda", dtype=dtype), torch.empty((0, 16), device="cuda", dtype=dtype)
        assert isam.linear(x, none).shape == (5, 0)
        assert (isam.linear_backward(x, none, torch.empty((5, 0), device="cuda", dtype=dtype))[0] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", ["none", "sigmoid", "silu", "gelu"])
@pytest.mark.parametrize("K,N", [(16, 8), (15, 7), (300, 300), (512, 512), (4096, 1024)])
def test_gradient_of_no_rows(K, N, name, dtype):
    e, W = torch.empty((0, K), device="cuda", dtype=dtype), torch.ones((N, K), device="cuda", dtype=dtype)
    dW, db = torch.full((N, K), 7.0, device="cuda", dtype=dtype), torch.full((N,), 7.0, device="cuda")
    dx, _, _ = isam.linear_backward(e, W, torch.empty((0, N), device="cuda", dtype=dtype), bias=torch.ones(N, device="cuda"), activation=name,
                                    dW=dW, dbias=db)
    assert dx.shape == (0, K) and (dW == 0).all() and (db == 0).all()


@pytest.mark.parametrize("name", ["none", "silu", "gelu"])
@pytest.mark.parametrize("M,K,N", [(5, 40, 30), (100, 40, 30)])
def test_gradient_against_differences(M, K, N, name):
    # central differences, step 2^-6: third-order terms below 2^-12 of the terms, rounding 2^-22 2^6 of the sums
    x = inputs(M, K, N, torch.float32, seed=M)
    grads = dict(zip(("x", "W", "bias"), isam.linear_backward(x["x"], x["W"], x["dout"], bias=x["bias"], activation=name)))
    g, step = torch.Generator(device="cuda").manual_seed(5), 2.0 ** -6
    for k, d in grads.items():
        v = torch.randn(x[k].shape, generator=g, device="cuda")
        side = []
        for s in (step, -step):
            y = {**x, k: x[k] + s * v}
            side.append(float((isam.linear(y["x"], y["W"], bias=y["bias"], activation=name).double() * x["dout"].double()).sum()))
        terms = d.double() * v.double()
        size = float((isam.linear(x["x"], x["W"], bias=x["bias"], activation=name).double() * x["dout"].double()).abs().sum())
        assert abs((side[0] - side[1]) / (2 * step) - float(terms.sum())) <= 2.0 ** -10 * float(terms.abs().sum()) + 2.0 ** -16 * size, k


@DTYPES
def test_infinite_values_stay_in_their_rows(dtype):
    x = inputs(130, 64, 72, dtype)
    x["x"][7] = float("nan")
    x["x"][100, 3] = float("inf")
    out = isam.linear(x["x"], x["W"], bias=x["bias"], activation="silu", residual=x["residual"])
    rows = torch.ones(130, dtype=torch.bool, device="cuda")
    rows[7] = rows[100] = False
    assert torch.isnan(out[7]).all() and torch.isfinite(out[rows].float()).all()


def test_streams_and_graph_replays():
    for M in (4, 200):
        x = inputs(M, 72, 80, torch.bfloat16, seed=M)
        code = isam.ISAM_BF16
        out, dx, dW, db = (torch.empty_like(x[k]) for k in ("dout", "x", "W", "bias"))
        w1 = torch.empty(max(1, isam.linear_workspace_size(M, 72, 80, code)), device="cuda", dtype=torch.uint8)
        w2 = torch.empty(isam.linear_backward_workspace_size(M, 72, 80, code), device="cuda", dtype=torch.uint8)

        def both(out, dx, dW, db):
            isam.linear(x["x"], x["W"], bias=x["bias"], activation="gelu", residual=x["residual"], out=out, workspace=w1)
            isam.linear_backward(x["x"], x["W"], x["dout"], bias=x["bias"], activation="gelu", dx=dx, dW=dW, dbias=db, workspace=w2)

        both(out, dx, dW, db)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both(out, dx, dW, db)
        for i in range(3):
            x["x"].copy_(torch.randn((M, 72), generator=torch.Generator().manual_seed(i)).to(torch.bfloat16))
            ref = tuple(torch.empty_like(t) for t in (out, dx, dW, db))
            both(*ref)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip((out, dx, dW, db), ref):
                assert torch.equal(a, b)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            other = isam.linear(x["x"], x["W"], bias=x["bias"], activation="gelu", residual=x["residual"])
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(other, out)


def test_refusals():
    x = inputs(40, 64, 72, torch.float32)
    for kw in (dict(bias=x["bias"][:5]), dict(residual=x["residual"][:5]), dict(activation="relu"), dict(out=torch.empty((40, 71), device="cuda"))):
        with pytest.raises(ValueError):
            isam.linear(x["x"], x["W"], **kw)
    for kw in (dict(bias=x["bias"].double()), dict(residual=x["residual"].bfloat16())):
        with pytest.raises(TypeError):
            isam.linear(x["x"], x["W"], **kw)
    with pytest.raises(ValueError):
        isam.linear(x["x"][:, :5], x["W"])
    with pytest.raises(TypeError):
        isam.linear(x["x"].half(), x["W"].half())
    with pytest.raises(ValueError):
        isam.linear(x["x"].cpu(), x["W"].cpu())
    with pytest.raises(isam.IsamError):          # a residual that is out shifted by a row
        r = torch.zeros((41, 72), device="cuda")
        isam.linear(x["x"], x["W"], residual=r[1:], out=r[:40])
    with pytest.raises(isam.IsamError):
        isam.linear_backward(x["x"], x["W"], x["dout"], dx=x["x"])
    with pytest.raises(isam.IsamError) as e:
        isam.linear_backward(x["x"], x["W"], x["dout"], workspace=torch.empty(16, device="cuda", dtype=torch.uint8))
    assert e.value.status == 3


@DTYPES
@pytest.mark.parametrize("M,K,N", [(17, 1024, 96), (31, 130, 50), (32, 1000, 4001), (33, 512, 17), (47, 33, 129), (48, 1365, 15), (49, 200, 333),
                                   (63, 1024, 100), (64, 1024, 512), (64, 1023, 70), (50, 2048, 40), (64, 4096, 200), (130, 4100, 72),
                                   (65, 8192, 64), (20, 6001, 333)])
def test_rows_between_few_and_tiles(M, K, N, dtype):
    """Up to 64 rows over little work, and deep products of few tiles: their own ways."""
    for i, name in enumerate(ACTS):
        compare(inputs(M, K, N, dtype, seed=M + i, bias=i != 1, residual=i != 2), name, backward=i == 3)


@DTYPES
@pytest.mark.parametrize("M,K,N", [(17, 1024, 96), (64, 1024, 512), (64, 4096, 200), (33, 1001, 65)])
def test_workspace_for_unaligned_rows_serves_aligned_ones(M, K, N, dtype):
    x = inputs(M, K, N, dtype, seed=K)
    code = 1 if dtype is torch.bfloat16 else 0
    room = torch.empty(max(isam.linear_workspace_size(M, K, N, code, aligned=False), 1), dtype=torch.uint8, device="cuda")
    check(isam.linear(x["x"], x["W"], bias=x["bias"], activation="gelu", residual=x["residual"], workspace=room), reference(x, "gelu")["out"], "out")
