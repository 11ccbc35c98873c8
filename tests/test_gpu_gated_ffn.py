"""GPU parity of the gated feed-forward block and its gradient against the formulas in 64 bits.

Tolerances are error bounds formed beside the 64-bit results, u = 2^-24.  A projection over K is good
to (K / 8 + 32) u of its sum of absolute products (sixteen products to an addition; fp32 products are formed
to about 2^-22); the activations and their slopes (at most 1.13 in slope themselves) add 32 u relative,
of 1 + |g|; dG and dU are rounded to bf16 as operands (half a unit in the last of 8 bits: up to 2^-8), sums
over M or 2F as over K; bf16 outputs add another such rounding.  Besides, the relative norm error of a result
of 256 values or more stays below 4e-3 for bf16 (the errors of one rounding have a norm of about 1.7e-3, of two
2.4e-3) and 2e-6 for fp32."""
import math

import pytest
import torch

import paper_1810_09958_amd as isam

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
OPERAND = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
NORM = {torch.float32: 2e-6, torch.bfloat16: 4e-3}


def inputs(M, K, F, dtype, seed=0, bias=True):
    g = torch.Generator().manual_seed(seed)
    return dict(x=torch.randn((M, K), generator=g).to(dtype).cuda(),
                W=(torch.randn((2 * F, K), generator=g) / math.sqrt(K)).to(dtype).cuda(),
                bias=(torch.randn(2 * F, generator=g) * 0.3).cuda() if bias else None,
                dout=torch.randn((M, F), generator=g).to(dtype).cuda())


def act(name, g):
    if name == "gelu":
        cdf = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    z, w = torch.sigmoid(g), torch.sigmoid(-g)
    return (z, z * w) if name == "sigmoid" else (g * z, z * (1 + g * w))


def mm(a, b):
    return torch.matmul(a.contiguous(), b.contiguous())


def reference(x, name):
    X, W, do = x["x"].double(), x["W"].double(), x["dout"].double()
    F, (M, K) = W.shape[0] // 2, X.shape
    b = x["bias"].double() if x["bias"] is not None else torch.zeros(2 * F, device=X.device, dtype=torch.float64)
    gu, s_gu = mm(X, W.t()) + b, mm(X.abs(), W.abs().t()) + b.abs()
    e_gu = (K / 8 + 32) * U * s_gu
    g, u, e_g, e_u = gu[:, :F], gu[:, F:], e_gu[:, :F], e_gu[:, F:]
    s, ds = act(name, g)
    e_s = 1.13 * e_g + 32 * U * (1 + g.abs())
    e_ds = e_g + 32 * U * (1 + g.abs())
    out = dict(out=(s * u, e_s * u.abs() + s.abs() * e_u + e_s * e_u + 2 * U * (s * u).abs()))
    d = torch.cat((do * u * ds, do * s), 1)
    e_d = torch.cat((do.abs() * (e_u * ds.abs() + u.abs() * e_ds + e_u * e_ds), do.abs() * e_s), 1) + 4 * U * d.abs()
    out["dbias"] = (d.sum(0), e_d.sum(0) + (M / 64 + 64) * U * d.abs().sum(0))
    r = OPERAND[x["x"].dtype]
    e_r = e_d + r * (d.abs() + e_d)
    out["dx"] = (mm(d, W), mm(e_r + (2 * F / 8 + 32) * U * d.abs(), W.abs()))
    out["dW"] = (mm(d.t(), X), mm((e_r + (M / 8 + 32) * U * d.abs()).t(), X.abs()))
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
    check(isam.gated_ffn(x["x"], x["W"], bias=x["bias"], activation=name), ref["out"], "out")
    if backward:
        got = dict(zip(("dx", "dW", "dbias"), isam.gated_ffn_backward(x["x"], x["W"], x["dout"], bias=x["bias"], activation=name)))
        for k, v in got.items():
            if v is not None:
                check(v, ref[k], k)


ACTS = ("sigmoid", "silu", "gelu")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,K,F", [(1, 64, 64), (1, 1, 1), (2, 8, 16), (3, 1000, 17), (7, 33, 100), (16, 4096, 48), (17, 64, 64),
                                   (1, 5000, 333)])
def test_few_tokens(M, K, F, dtype):
    for i, name in enumerate(ACTS):
        compare(inputs(M, K, F, dtype, seed=M + i, bias=i != 1), name, backward=i == 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,K,F", [(33, 64, 32), (64, 128, 96), (65, 72, 33), (100, 200, 65), (200, 520, 40), (130, 7, 9),
                                   (64, 1, 64), (300, 511, 77), (1000, 96, 1)])
def test_small_tiles(M, K, F, dtype):
    for i, name in enumerate(ACTS):
        compare(inputs(M, K, F, dtype, seed=M + i, bias=i != 1), name)


@pytest.mark.parametrize("M,K,F", [(1, 210, 76), (2, 64, 128), (5, 333, 1001), (16, 1000, 31), (16, 72, 515)])
def test_gradient_of_few_tokens_rounds_once(M, K, F):
    # Over few rows the rounding of an operand is not averaged out: dx and dW are within one rounding of the
    # output, at most 2^-9 of each value and so of the norm, and what two terms of 8 bits lose, below 2^-13
    for i, name in enumerate(ACTS):
        x = inputs(M, K, F, torch.bfloat16, seed=M + i, bias=i != 1)
        ref = reference(x, name)
        got = isam.gated_ffn_backward(x["x"], x["W"], x["dout"], bias=x["bias"], activation=name)
        for k, v in zip(("dx", "dW"), got):
            check(v, ref[k], k)
            assert float((v.double() - ref[k][0]).norm()) <= (2.0 ** -9 + 2.0 ** -13) * float(ref[k][0].norm()), k
        # alone, and into strided outputs, the same bits
        dx = torch.empty((M, K + 5), device="cuda", dtype=torch.bfloat16)[:, 3:3 + K]
        isam.gated_ffn_backward(x["x"], x["W"], x["dout"], bias=x["bias"], activation=name, dx=dx)
        assert torch.equal(dx, got[0])


@pytest.mark.parametrize("M,K,F", [(600, 700, 900), (2000, 130, 1501), (40, 1700, 50), (333, 1537, 513), (1000, 24, 777),
                                   (500, 511, 771), (1025, 80, 1031), (17, 1536, 3000)])
def test_fp32_sizes(M, K, F):
    # both sides of the rule between the block's own fp32 kernel and the library's product
    for i, name in enumerate(ACTS):
        compare(inputs(M, K, F, torch.float32, seed=M + i, bias=i != 1), name)


@pytest.mark.parametrize("M,K,F", [(1024, 64, 2048), (1000, 200, 2111), (1100, 136, 2100), (1023, 65, 2050)])
def test_middle_tiles(M, K, F):
    for i, name in enumerate(ACTS):
        compare(inputs(M, K, F, torch.bfloat16, seed=M + i, bias=i != 1), name)


@pytest.mark.parametrize("M,K,F", [(2048, 128, 4096), (2100, 200, 4000), (4000, 328, 2047), (2047, 63, 4100)])
def test_large_tiles(M, K, F):
    for i, name in enumerate(ACTS):
        compare(inputs(M, K, F, torch.bfloat16, seed=M + i, bias=i != 1), name)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M", [5, 70, 1100])
def test_strides_and_alignment(M, dtype):
    K, F = 72, 2056 if M > 1000 else 41
    x = inputs(M, K, F, dtype, seed=M)
    ref = reference(x, "silu")

    def wide(t, off, pad):
        w = torch.full((t.shape[0], t.shape[1] + pad), 7.0, device="cuda", dtype=dtype)
        w[:, off:off + t.shape[1]] = t
        return w, w[:, off:off + t.shape[1]]

    for off, pad in ((8, 16), (3, 7)):           # aligned rows, and rows off 16 bytes
        (_, xs), (_, ws), (_, do) = wide(x["x"], off, pad), wide(x["W"], off, pad), wide(x["dout"], off, pad)
        (ow, out), (dxw, dx), (dww, dW) = wide(ref["out"][0].to(dtype) * 0, off, pad), wide(x["x"] * 0, off, pad), wide(x["W"] * 0, off, pad)
        isam.gated_ffn(xs, ws, bias=x["bias"], out=out)
        check(out, ref["out"], "out")
        _, _, db = isam.gated_ffn_backward(xs, ws, do, bias=x["bias"], dx=dx, dW=dW)
        for k, v in (("dx", dx), ("dW", dW), ("dbias", db)):
            check(v, ref[k], k)
        for w in (ow, dxw, dww):
            assert (w[:, :off] == 7).all() and (w[:, w.shape[1] - (pad - off):] == 7).all()
    # one operand aligned, the other not
    isam_out = isam.gated_ffn(wide(x["x"], 3, 7)[1], x["W"], bias=x["bias"])
    check(isam_out, ref["out"], "out")
    check(isam.gated_ffn(x["x"], wide(x["W"], 3, 7)[1], bias=x["bias"]), ref["out"], "out")


def test_empty():
    for dtype in (torch.float32, torch.bfloat16):
        x = inputs(0, 24, 16, dtype)
        assert isam.gated_ffn(x["x"], x["W"], bias=x["bias"]).shape == (0, 16)
        dx, dW, db = isam.gated_ffn_backward(x["x"], x["W"], x["dout"], bias=x["bias"])
        assert dx.shape == (0, 24) and (dW == 0).all() and (db == 0).all()
        x = inputs(5, 24, 0, dtype)
        assert isam.gated_ffn(x["x"], x["W"]).shape == (5, 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", ACTS)
def test_saturated_gates(name, dtype):
    # gate projections far out on both sides: no NaN from 0 * inf
    for M in (4, 40):
        x = inputs(M, 32, 24, dtype, seed=M)
        x["bias"][:8] = -1e4
        x["bias"][8:16] = 1e4
        compare(x, name)


@pytest.mark.parametrize("M", [3, 40, 1100])
def test_bad_row_stays_with_itself(M):
    x = inputs(M, 64, 2048 if M > 1000 else 40, torch.bfloat16, seed=1)
    good = isam.gated_ffn(x["x"], x["W"])
    x["x"][1, 5] = float("nan")
    bad = isam.gated_ffn(x["x"], x["W"])
    assert torch.isnan(bad[1].float()).all()
    keep = [i for i in range(M) if i != 1]
    assert torch.equal(bad[keep], good[keep])


@pytest.mark.parametrize("M,K,F,dtype", [(1100, 200, 2050, torch.bfloat16), (70, 72, 33, torch.bfloat16), (300, 511, 77, torch.float32)])
def test_repeats_bit_for_bit(M, K, F, dtype):
    x = inputs(M, K, F, dtype, seed=5)

    def both():
        return (isam.gated_ffn(x["x"], x["W"], bias=x["bias"]), *isam.gated_ffn_backward(x["x"], x["W"], x["dout"], bias=x["bias"]))

    first = both()
    for _ in range(4):
        for a, b in zip(first, both()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("name", ACTS)
def test_gradient_against_differences(name):
    # central differences of the fp32 forward pass along a random direction, step 2^-6: third-order term
    # below 2^-11 of the sums here, rounding about 2^-17
    x = inputs(40, 24, 20, torch.float32, seed=3)
    grads = dict(zip(("x", "W", "bias"), isam.gated_ffn_backward(x["x"], x["W"], x["dout"], bias=x["bias"], activation=name)))
    arg = {k: x[k] for k in ("x", "W", "bias")}

    def loss(a):
        return float((isam.gated_ffn(activation=name, **a).double() * x["dout"].double()).sum())

    g = torch.Generator(device="cuda").manual_seed(5)
    step = 2.0 ** -6
    for k, grad in grads.items():
        v = torch.randn(arg[k].shape, generator=g, device="cuda") * (0.2 if k == "W" else 1.0)
        diff = (loss({**arg, k: arg[k] + step * v}) - loss({**arg, k: arg[k] - step * v})) / (2 * step)
        prod = grad.double() * v.double()
        assert abs(diff - float(prod.sum())) <= 2.0 ** -9 * float(prod.abs().sum()), k


def test_graph_replays():
    M, K, F = 300, 100, 130
    for dtype, code in ((torch.bfloat16, 1), (torch.float32, 0)):
        x = inputs(M, K, F, dtype, seed=7)
        w1 = torch.empty(isam.gated_ffn_workspace_size(M, K, F, code), device="cuda", dtype=torch.uint8)
        w2 = torch.empty(isam.gated_ffn_backward_workspace_size(M, K, F, code), device="cuda", dtype=torch.uint8)
        out, dx, dW = torch.empty_like(x["dout"]), torch.empty_like(x["x"]), torch.empty_like(x["W"])
        db = torch.empty_like(x["bias"])

        def both():
            isam.gated_ffn(x["x"], x["W"], bias=x["bias"], out=out, workspace=w1)
            isam.gated_ffn_backward(x["x"], x["W"], x["dout"], bias=x["bias"], dx=dx, dW=dW, dbias=db, workspace=w2)

        both()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            both()
        for i in range(3):
            x["x"].copy_(torch.randn(x["x"].shape, generator=torch.Generator().manual_seed(i)))
            both()
            torch.cuda.synchronize()
            ref = [t.clone() for t in (out, dx, dW, db)]
            for t in (out, dx, dW, db):
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip((out, dx, dW, db), ref):
                assert torch.equal(a, b)


def test_refusals():
    x = inputs(40, 32, 16, torch.bfloat16)
    with pytest.raises(ValueError):
        isam.gated_ffn(x["x"], x["W"][:31])
    with pytest.raises(ValueError):
        isam.gated_ffn(x["x"], x["W"][:, :30])
    with pytest.raises(ValueError):
        isam.gated_ffn(x["x"], x["W"], activation="relu")
    with pytest.raises(ValueError):
        isam.gated_ffn(x["x"], x["W"], bias=x["bias"][:16])
    with pytest.raises(ValueError):
        isam.gated_ffn(x["x"].t(), x["W"])
    with pytest.raises(TypeError):
        isam.gated_ffn(x["x"], x["W"].float())
    with pytest.raises(TypeError):
        isam.gated_ffn_backward(x["x"], x["W"], x["dout"].float())
    with pytest.raises(isam.IsamError):
        isam.gated_ffn(x["x"], x["W"], out=x["x"][:, :16])
    with pytest.raises(isam.IsamError):
        isam.gated_ffn(x["x"][:, :0], x["W"][:, :0])
    y = inputs(40, 33, 16, torch.bfloat16)
    with pytest.raises(isam.IsamError) as e:     # copies need room
        isam.gated_ffn(y["x"], y["W"], workspace=torch.empty(8, device="cuda", dtype=torch.uint8))
    assert e.value.status == 3


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,K,F", [(130, 7, 9), (5, 7, 9), (130, 7, 40), (130, 1, 33), (300, 72, 41)])
def test_bad_row_stays_with_itself_in_dx(M, K, F, dtype):
    x = inputs(M, K, F, dtype, seed=2)
    good = isam.gated_ffn_backward(x["x"], x["W"], x["dout"], bias=x["bias"])[0]
    x["dout"][1] = float("nan")
    bad = isam.gated_ffn_backward(x["x"], x["W"], x["dout"], bias=x["bias"])[0]
    keep = [i for i in range(M) if i != 1]
    assert torch.isnan(bad[1].float()).all()
    assert torch.equal(bad[keep], good[keep])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_empty_block_has_zero_gradient(dtype):
    # no hidden values: the block gives [M][0], and nothing comes back through it
    for M in (0, 5, 40):
        x = inputs(M, 24, 0, dtype)
        dx = torch.full((M, 24), 7.0, device="cuda", dtype=dtype)
        got, dW, db = isam.gated_ffn_backward(x["x"], x["W"], x["dout"], bias=x["bias"], dx=dx)
        assert got is dx and (dx == 0).all() and dW.shape == (0, 24) and db.shape == (0,)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,K,F", [(5, 72, 41), (70, 72, 40), (600, 700, 900), (40, 24, 0)])
def test_parts_of_the_gradient(M, K, F, dtype):
    # what is asked for alone is what the whole call gives, bit for bit; the rest is None
    x = inputs(M, K, F, dtype, seed=3)
    call = lambda **kw: isam.gated_ffn_backward(x["x"], x["W"], x["dout"], bias=x["bias"], **kw)
    dx, dW, db = call()
    a, b, c = call(return_dW=False)
    assert torch.equal(a, dx) and b is None and torch.equal(c, db)
    a, b, c = call(return_dx=False)
    assert a is None and torch.equal(b, dW) and torch.equal(c, db)
    a, b, c = call(return_dx=False, return_dW=False)
    assert a is None and b is None and torch.equal(c, db)
    if F:
        with pytest.raises(isam.IsamError):      # nothing left to form
            isam.gated_ffn_backward(x["x"], x["W"], x["dout"], return_dx=False, return_dW=False)


# Both sides of the limits between the tiles: one round of small tiles or more, and large tiles whose rounds
# are nearly full or nearly empty; whole and ragged rows, columns and K.
@pytest.mark.parametrize("M,K,F", [(512, 72, 2048), (513, 72, 2048), (1000, 63, 1030), (2000, 64, 512), (1537, 64, 4096),
                                   (1700, 65, 4095), (2047, 63, 4096), (2049, 128, 4096), (2900, 40, 4001), (3200, 64, 4097)])
def test_tile_limits(M, K, F):
    for i, name in enumerate(ACTS):
        compare(inputs(M, K, F, torch.bfloat16, seed=M + i, bias=i != 1), name)
