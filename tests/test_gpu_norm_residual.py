"""GPU parity of the gated residual norm and its gradient against the formulas in 64 bits.

Tolerances are error bounds formed beside the 64-bit results, u = 2^-24.  A sum of n squares over
the threads of a row is good to (n / 64 + 16) u, its root to half of that; products add u each.
A sum over rows is a chain of at most rows / 64 + 64 additions.  bf16 outputs add half a unit in
their last place."""
import pytest
import torch

import paper_1810_09958_amd as isam

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}


def inputs(R, D, G, dtype, seed=0, post=True, gate=True, block=True):
    g = torch.Generator().manual_seed(seed)

    def m(rows, scale=1.0):
        return (torch.randn((rows, D), generator=g) * scale).to(dtype).cuda()

    return dict(x=m(R) if block else None, r=m(R, 2.0), gate=m(G, 0.5) if gate else None,
                w_post=(torch.rand(D, generator=g) + 0.5).cuda() if post else None,
                w_pre=(torch.rand(D, generator=g) + 0.5).cuda(), dy=m(R), dr_out=m(R))


def reference(x, scale, eps, forward):
    f = {k: (v.cpu().double() if v is not None else None) for k, v in x.items()}
    R, D = f["r"].shape
    k = (D / 64 + 16) * U + 8 * U                       # relative error of a norm's factor
    q, e_q = torch.ones(R, 1, dtype=torch.float64), 0.0
    if f["x"] is not None:
        if f["w_post"] is not None:
            q, e_q = 1 / torch.sqrt((f["x"] ** 2).mean(1, keepdim=True) + eps), k
        xn = f["x"] * q
        w = f["w_post"] if f["w_post"] is not None else 1.0
        u = xn * w
        G = f["gate"].shape[0] if f["gate"] is not None else 1
        gate = scale * (f["gate"].repeat_interleave(R // G, 0) if f["gate"] is not None else torch.ones(R, D, dtype=torch.float64))
    if forward:
        r, e_r = f["r"], torch.zeros_like(f["r"])
        if f["x"] is not None:
            t = gate * u
            r, e_r = f["r"] + t, (e_q + 4 * U) * t.abs()
            e_r = e_r + U * r.abs()
        p = 1 / torch.sqrt((r ** 2).mean(1, keepdim=True) + eps)
        y = r * p * f["w_pre"]
        e_p = k + (e_r ** 2).mean(1, keepdim=True).sqrt() * p
        return dict(r_out=(r, e_r), y=(y, e_r * p * f["w_pre"].abs() + (e_p + 4 * U) * y.abs()))
    r = f["r"]
    p = 1 / torch.sqrt((r ** 2).mean(1, keepdim=True) + eps)
    t = f["dy"] * f["w_pre"]
    c, c_abs = p ** 3 * (t * r).mean(1, keepdim=True), p ** 3 * (t * r).abs().mean(1, keepdim=True)
    d0 = f["dr_out"] if f["dr_out"] is not None else 0.0
    dr = d0 + p * t - c * r
    e_dr = 4 * (k + 4 * U) * ((p * t).abs() + c_abs * r.abs()) + 2 * U * (dr.abs() + abs(d0))
    chain = (R / 64 + 64) * U
    terms = f["dy"] * p * r
    out = dict(dr=(dr, e_dr), dw_pre=(terms.sum(0), (k + 4 * U + chain) * terms.abs().sum(0)))
    if f["x"] is None:
        return out
    du, e_du = gate * dr, gate.abs() * (e_dr + 4 * U * dr.abs())
    if f["gate"] is not None:
        terms, e_t = scale * u * dr, (scale * u).abs() * (e_dr + (e_q + 4 * U + chain) * dr.abs())
        out["dgate"] = (terms.view(G, R // G, D).sum(1), e_t.view(G, R // G, D).sum(1))
    if f["w_post"] is None:
        out["dx"] = (du, e_du)
        return out
    out["dw_post"] = ((du * xn).sum(0), (xn.abs() * (e_du + (k + 4 * U + chain) * du.abs())).sum(0))
    v, e_v = du * w, w * (e_du + 2 * U * du.abs())
    m, m_abs = q ** 3 * (v * f["x"]).mean(1, keepdim=True), q ** 3 * (v * f["x"]).abs().mean(1, keepdim=True)
    e_m = q ** 3 * (e_v * f["x"].abs()).mean(1, keepdim=True) + 4 * (k + 4 * U) * m_abs
    dx = q * v - m * f["x"]
    out["dx"] = (dx, q * e_v + (k + 8 * U) * (q * v).abs() + f["x"].abs() * e_m + 4 * U * dx.abs())
    return out


def check(got, ref, name):
    val, bound = ref
    bound = bound + HALF[got.dtype] * val.abs() + 1e-30
    err = (got.cpu().double() - val).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / bound).max()):.2f} bounds"


def compare(x, scale=0.7, eps=1e-6, **kw):
    opt = dict(w_pre=x["w_pre"], w_post=x["w_post"], gate=x["gate"], scale=scale, eps=eps)
    r_out, y = isam.norm_residual(x["x"], x["r"], **opt)
    ref = reference(x, scale, eps, True)
    check(r_out, ref["r_out"], "r_out")
    check(y, ref["y"], "y")
    got = dict(zip(("dx", "dr", "dgate", "dw_post", "dw_pre"),
                   isam.norm_residual_backward(x["x"], x["r"], x["dy"], dr_out=x["dr_out"], **opt, **kw)))
    ref = reference(x, scale, eps, False)
    assert {k for k, v in got.items() if v is not None} == set(ref)
    for k, v in ref.items():
        check(got[k], v, k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [1, 2, 7, 8, 63, 64, 200, 511, 513, 1024, 1030, 2047, 2050, 4096, 4100, 8200, 10001, 16384])
def test_widths(D, dtype):
    compare(inputs(9, D, 1, dtype, seed=D))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,G", [(1, 1), (2, 2), (5, 1), (24, 3), (64, 64), (3000, 1), (3000, 3000), (3000, 10), (9000, 3000),
                                 (6000, 1500)])
def test_rows_and_gates(R, G, dtype):
    compare(inputs(R, 72, G, dtype, seed=R))


@pytest.mark.parametrize("D", [600, 3000, 9000])
def test_many_gate_rows_of_long_rows(D):
    compare(inputs(2600, D, 1300, torch.bfloat16, seed=D))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [40, 1000, 5000])
def test_optional_arguments(D, dtype):
    for post in (False, True):
        for gate in (False, True):
            for dr in (False, True):
                x = inputs(33, D, 11, dtype, seed=D, post=post, gate=gate)
                if not dr:
                    x["dr_out"] = None
                compare(x)
    x = inputs(33, D, 1, dtype, seed=D, post=False, gate=False, block=False)
    compare(x)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_in_place(dtype):
    R, D = 40, 203
    x = inputs(R, D, 4, dtype, seed=1)

    def wide(t, fill=7.0):
        w = torch.full((R, D + 9), fill, device="cuda", dtype=dtype)
        w[:, 4:4 + D] = t
        return w, w[:, 4:4 + D]

    ref_f, ref_b = reference(x, 0.7, 1e-6, True), reference(x, 0.7, 1e-6, False)
    opt = dict(w_pre=x["w_pre"], w_post=x["w_post"], gate=x["gate"], scale=0.7)
    (_, xs), (rw, rs), (yw, ys) = wide(x["x"]), wide(x["r"]), wide(0.0)
    r_out, _ = isam.norm_residual(xs, rs, r_out=rs, y=ys, **opt)
    assert r_out is rs
    check(rs, ref_f["r_out"], "r_out")
    check(ys, ref_f["y"], "y")
    (_, r2), (_, dy), (dw, dr), (xw, dx) = wide(x["r"]), wide(x["dy"]), wide(x["dr_out"]), wide(0.0)
    isam.norm_residual_backward(xs, r2, dy, dr_out=dr, dr=dr, dx=dx, **opt)
    check(dr, ref_b["dr"], "dr")
    check(dx, ref_b["dx"], "dx")
    for w in (rw, yw, dw, xw):
        assert (w[:, :4] == 7).all() and (w[:, 4 + D:] == 7).all()


def test_empty():
    x = inputs(0, 16, 0, torch.float32)
    opt = dict(w_pre=x["w_pre"], w_post=x["w_post"])
    r_out, y = isam.norm_residual(x["x"], x["r"], **opt)
    assert r_out.shape == y.shape == (0, 16)
    dgate = torch.full((3, 16), 7.0, device="cuda")
    out = isam.norm_residual_backward(x["x"], x["r"], x["dy"], gate=torch.ones((3, 16), device="cuda"), dgate=dgate, **opt)
    assert out[0].shape == (0, 16) and all((t == 0).all() for t in out[2:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_extreme_rows(dtype):
    # a row of zeros (the norm of nothing is nothing), rows of tiny and of large values
    x = inputs(6, 520, 1, dtype, seed=3)
    x["x"][0] = 0
    x["r"][1] = 0
    x["x"][1] = 0
    x["x"][2] *= 1e-15
    x["x"][3] *= 1e15
    x["r"][4] *= 1e15
    compare(x)
    # a bad row stays with itself
    good = isam.norm_residual(x["x"], x["r"], w_pre=x["w_pre"], w_post=x["w_post"], gate=x["gate"])
    x["x"][5, 3] = float("nan")
    out = isam.norm_residual(x["x"], x["r"], w_pre=x["w_pre"], w_post=x["w_post"], gate=x["gate"])
    for a, b in zip(good, out):
        assert torch.equal(a[:5], b[:5]) and torch.isnan(b[5].float()).all()


@pytest.mark.parametrize("R,D,G", [(3000, 520, 1), (3000, 2100, 30), (700, 4100, 700)])
def test_repeats_bit_for_bit(R, D, G):
    x = inputs(R, D, G, torch.bfloat16, seed=5)
    opt = dict(w_pre=x["w_pre"], w_post=x["w_post"], gate=x["gate"], dr_out=x["dr_out"])
    first = isam.norm_residual_backward(x["x"], x["r"], x["dy"], **opt)
    for _ in range(4):
        for a, b in zip(first, isam.norm_residual_backward(x["x"], x["r"], x["dy"], **opt)):
            assert torch.equal(a, b)


def test_gradient_against_differences():
    # central differences of the forward pass, step 2^-6: third-order term below 2^-11 of the sums here
    R, D, G, step = 12, 96, 3, 2.0 ** -6
    x = inputs(R, D, G, torch.float32, seed=8)
    arg = {k: x[k] for k in ("x", "r", "gate", "w_post", "w_pre")}
    r_out, _ = isam.norm_residual(scale=0.7, **arg)
    grads = dict(zip(("x", "r", "gate", "w_post", "w_pre"), isam.norm_residual_backward(
        x["x"], r_out, x["dy"], dr_out=x["dr_out"], scale=0.7, gate=x["gate"], w_post=x["w_post"], w_pre=x["w_pre"])))

    def loss(a):
        r_out, y = isam.norm_residual(scale=0.7, **a)
        return float((y.double() * x["dy"].double()).sum() + (r_out.double() * x["dr_out"].double()).sum())

    g = torch.Generator(device="cuda").manual_seed(5)
    for name, grad in grads.items():
        v = torch.randn(arg[name].shape, generator=g, device="cuda")
        diff = (loss({**arg, name: arg[name] + step * v}) - loss({**arg, name: arg[name] - step * v})) / (2 * step)
        prod = grad.double() * v.double()
        assert abs(diff - float(prod.sum())) <= 2.0 ** -9 * float(prod.abs().sum()), name


def test_long_offsets():
    # leading dimensions that take the last rows past 2^31 elements
    R, D, ld = 260, 64, (1 << 31) // 256
    x = inputs(R, D, 1, torch.bfloat16, seed=6)
    big = torch.empty(((R - 1) * ld + D,), device="cuda", dtype=torch.bfloat16)
    far = big.as_strided((R, D), (ld, 1))
    far.copy_(x["x"])
    x["x"] = far
    compare(x)


def test_graph_replays():
    R, D = 3000, 520
    x = inputs(R, D, 1, torch.bfloat16, seed=7)
    opt = dict(w_pre=x["w_pre"], w_post=x["w_post"], gate=x["gate"])
    ws = torch.empty(isam.norm_residual_backward_workspace_size(R, D, 1, 1), device="cuda", dtype=torch.uint8)
    bufs = [torch.empty_like(x["x"]), torch.empty_like(x["x"]), torch.empty_like(x["x"]), torch.empty_like(x["x"]),
            torch.empty_like(x["gate"]), torch.empty_like(x["w_post"]), torch.empty_like(x["w_pre"])]

    def both():
        isam.norm_residual(x["x"], x["r"], r_out=bufs[0], y=bufs[1], **opt)
        isam.norm_residual_backward(x["x"], bufs[0], x["dy"], dr_out=x["dr_out"], dx=bufs[2], dr=bufs[3], dgate=bufs[4],
                                    dw_post=bufs[5], dw_pre=bufs[6], workspace=ws, **opt)

    both()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for i in range(3):
        x["x"].copy_(torch.randn(x["x"].shape, generator=torch.Generator().manual_seed(i)))
        both()
        torch.cuda.synchronize()
        ref = [b.clone() for b in bufs]
        for b in bufs:
            b.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(bufs, ref):
            assert torch.equal(a, b)


def test_refusals():
    x = inputs(12, 32, 3, torch.float32)
    opt = dict(w_pre=x["w_pre"], w_post=x["w_post"], gate=x["gate"])
    for kw in (dict(gate=x["gate"][:, :5]), dict(gate=torch.ones((5, 32), device="cuda")), dict(w_pre=x["w_pre"][:4]),
               dict(y=torch.empty((12, 31), device="cuda"))):
        with pytest.raises(ValueError):
            isam.norm_residual(x["x"], x["r"], **{**opt, **kw})
    for kw in (dict(gate=x["gate"].bfloat16()), dict(w_post=x["w_post"].bfloat16())):
        with pytest.raises(TypeError):
            isam.norm_residual(x["x"], x["r"], **{**opt, **kw})
    with pytest.raises(TypeError):
        isam.norm_residual(x["x"].bfloat16(), x["r"], **opt)
    for kw in (dict(y=x["x"]), dict(r_out=x["x"]), dict(eps=-1.0), dict(scale=float("nan"))):
        with pytest.raises(isam.IsamError):
            isam.norm_residual(x["x"], x["r"], **{**opt, **kw})
    with pytest.raises(isam.IsamError):           # a gate without a block output
        isam.norm_residual(None, x["r"], **opt)
    with pytest.raises(isam.IsamError) as e:
        isam.norm_residual(None, torch.zeros((1, 16385), device="cuda"), w_pre=torch.ones(16385, device="cuda"))
    assert e.value.status == 2
    with pytest.raises(isam.IsamError) as e:
        isam.norm_residual_backward(x["x"], x["r"], x["dy"], workspace=torch.empty(8, device="cuda", dtype=torch.uint8), **opt)
    assert e.value.status == 3
