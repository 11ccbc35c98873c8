"""GPU parity of the linear GRU and its gradient against the recurrence in 64 bits.

Tolerances are running error bounds formed beside the 64-bit results.  u = 2^-24; a gate value
carries a relative error of at most 32 u (its exponential's argument, up to 20 in magnitude here, is
rounded at 2^-24 relative: 29 u; a few more for the sum, the reciprocal and the product), so a step
adds at most 32 u (|z h| + |(1-z) n|) to what z leaves of the error before it; composing steps in
another order rounds the same products.  bf16 outputs add half a unit in their last place."""
import numpy as np
import pytest
import torch

import paper_1810_09958_amd as isam

U = 2.0 ** -24
STEP = 32 * U
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}    # rounding of an output, relative (with slack)


def inputs(T, B, H, dtype, seed=0, batch_first=False, reset=None, train=True):
    g = torch.Generator().manual_seed(seed)

    def rows(w):
        t = torch.randn((B, T, w) if batch_first else (T, B, w), generator=g).to(dtype).cuda()
        return t.transpose(0, 1) if batch_first else t

    x = dict(gx=rows(2 * H), bias=torch.cat((torch.rand(H, generator=g) * 6 - 1, torch.randn(H, generator=g) * 0.2)).cuda(),
             h0=torch.randn((B, H), generator=g).cuda(), reset=None)
    if reset is not None:
        r = torch.rand((B, T) if batch_first else (T, B), generator=g) < reset
        r = r.cuda()
        x["reset"] = r.t() if batch_first else r
    if train:
        x["dh_seq"] = rows(H)
        x["dh_T"] = torch.randn((B, H), generator=g).cuda()
    return x


def reference(x, candidate, H):
    """64-bit results and their bounds: dicts of (value, bound)."""
    f = {k: (v.cpu().double() if v is not None and v.is_floating_point() else v) for k, v in x.items()}
    bias = f["bias"] if f["bias"] is not None else torch.zeros(2 * H, dtype=torch.float64)
    gx = f["gx"] + bias
    T, B = gx.shape[:2]
    z = torch.sigmoid(gx[..., :H])
    w = torch.sigmoid(-gx[..., :H])
    v = gx[..., H:]
    n = torch.tanh(v) if candidate == "tanh" else v
    en = 4 * U + STEP * n.abs()                        # tanh: absolute error of a few u
    a = z.clone()
    if x["reset"] is not None:
        a[x["reset"].cpu().bool()] = 0
    h = f["h0"] if f["h0"] is not None else torch.zeros((B, H), dtype=torch.float64)
    eh = torch.zeros_like(h)
    hs, ehs, prev, eprev = [], [], [], []
    for t in range(T):
        prev.append(torch.where(a[t] == 0, 0.0, h))
        eprev.append(torch.where(a[t] == 0, 0.0, eh))
        h, eh = a[t] * h + w[t] * n[t], a[t] * eh + STEP * ((a[t] * h).abs() + (w[t] * n[t]).abs()) + w[t] * en[t]
        hs.append(h)
        ehs.append(eh)
    out = dict(h_T=(h, eh))
    if T:
        out["h_seq"] = (torch.stack(hs), torch.stack(ehs))
    if "dh_seq" not in x:
        return out
    e = f["dh_T"] if f["dh_T"] is not None else torch.zeros((B, H), dtype=torch.float64)
    ee = torch.zeros_like(e)
    dg, edg = torch.zeros_like(gx), torch.zeros_like(gx)
    for t in range(T - 1, -1, -1):
        dh = f["dh_seq"][t] if f["dh_seq"] is not None else 0
        d, ed = dh + e, ee + U * (dh + e).abs()
        s = z[t] * w[t]
        dg[t, :, :H] = d * (prev[t] - n[t]) * s
        edg[t, :, :H] = s * (ed * (prev[t] - n[t]).abs() + d.abs() * (eprev[t] + en[t] + 3 * STEP * (prev[t].abs() + n[t].abs())))
        slope = (1 - n[t] ** 2) if candidate == "tanh" else torch.ones_like(d)
        dg[t, :, H:] = d * w[t] * slope
        edg[t, :, H:] = w[t] * (ed * slope.abs() + d.abs() * (2 * STEP + 2 * en[t] * n[t].abs() * (candidate == "tanh")))
        e, ee = a[t] * d, a[t] * (ed + STEP * d.abs())
    out["dgx"], out["dh0"] = (dg, edg), (e, ee)
    out["dbias"] = (dg.sum((0, 1)), edg.sum((0, 1)) + 64 * U * dg.abs().sum((0, 1)))
    return out


def check(got, ref, name):
    val, bound = ref
    bound = bound + HALF[got.dtype] * val.abs() + 1e-30
    err = (got.cpu().double() - val).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / bound).max()):.2f} bounds"


def run(x, candidate, train=True):
    T, B, H2 = x["gx"].shape
    states = torch.full(isam.linear_gru_states_shape(T, B, H2 // 2), float("nan"), device="cuda")
    out = {}
    out["h_seq"], out["h_T"] = isam.linear_gru(x["gx"], bias=x["bias"], h0=x["h0"], reset=x["reset"], candidate=candidate,
                                               states=states)
    if train:
        out["dgx"], out["dh0"], out["dbias"] = isam.linear_gru_backward(
            x["gx"], x["dh_seq"], states=states, bias=x["bias"], reset=x["reset"], candidate=candidate, dh_T=x["dh_T"])
    torch.cuda.synchronize()
    return {k: v for k, v in out.items() if v is not None}   # (no dbias without a bias)


def compare(x, candidate, train=True):
    ref = reference(x, candidate, x["gx"].shape[2] // 2)
    for k, v in run(x, candidate, train).items():
        if k in ref:
            check(v, ref[k], k)


pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 31, 64, 65, 255, 256, 257, 700])
def test_lengths(T, dtype):
    compare(inputs(T, 3, 72, dtype, seed=T, reset=0.05 if T % 2 else None), "tanh" if T % 3 else "linear")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H", [1, 3, 8, 31, 63, 65, 100, 333])
def test_widths(H, dtype):
    compare(inputs(300, 2, H, dtype, seed=H, reset=0.01), "tanh")
    compare(inputs(20, 5, H, dtype, seed=H), "linear")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,B,H,reset", [(1024, 1, 64, None), (1500, 1, 200, 0.002), (5000, 2, 40, 0.001), (9000, 1, 33, None)])
def test_time_in_segments(T, B, H, reset, dtype):
    # few sequences and channels: time is cut into segments
    compare(inputs(T, B, H, dtype, seed=T, reset=reset), "tanh")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_batch_first_and_slices(dtype):
    compare(inputs(333, 4, 40, dtype, batch_first=True, reset=0.01), "tanh")
    compare(inputs(5, 4, 40, dtype, batch_first=True, reset=0.2), "tanh")
    # gates, states and gradients as slices of wider rows, off 16 bytes
    T, B, H = 300, 3, 37
    x = inputs(T, B, H, dtype, seed=3)
    wide = torch.zeros((T, B, 2 * H + 5), device="cuda", dtype=dtype)
    wide[..., 3:3 + 2 * H] = x["gx"]
    x["gx"] = wide[..., 3:3 + 2 * H]
    ref = reference(x, "tanh", H)
    hs = torch.full((T, B, H + 3), 7.0, device="cuda", dtype=dtype)
    dg = torch.full((T, B, 2 * H + 3), 7.0, device="cuda", dtype=dtype)
    states = torch.empty(isam.linear_gru_states_shape(T, B, H), device="cuda")
    isam.linear_gru(x["gx"], bias=x["bias"], h0=x["h0"], h_seq=hs[..., 1:1 + H], states=states)
    isam.linear_gru_backward(x["gx"], x["dh_seq"], states=states, bias=x["bias"], dh_T=x["dh_T"], dgx=dg[..., 2:2 + 2 * H])
    check(hs[..., 1:1 + H], ref["h_seq"], "h_seq")
    check(dg[..., 2:2 + 2 * H], ref["dgx"], "dgx")
    for t, lo, hi in ((hs, 1, 1 + H), (dg, 2, 2 + 2 * H)):     # nothing beside the rows is touched
        assert (t[..., :lo] == 7).all() and (t[..., hi:] == 7).all()


@pytest.mark.parametrize("T", [6, 300, 2100])
def test_optional_arguments(T):
    H = 24
    x = inputs(T, 2, H, torch.float32, seed=T)
    x["bias"] = x["h0"] = x["dh_T"] = None
    compare(x, "tanh")
    x = inputs(T, 2, H, torch.float32, seed=T)
    x["dh_seq"] = None
    compare(x, "tanh")
    hs, hT = isam.linear_gru(x["gx"], bias=x["bias"], h0=x["h0"], return_sequence=False)
    assert hs is None
    check(hT, reference(x, "tanh", H)["h_T"], "h_T")


def test_empty():
    x = inputs(0, 3, 16, torch.float32)
    states = torch.empty(isam.linear_gru_states_shape(0, 3, 16), device="cuda")
    hs, hT = isam.linear_gru(x["gx"], bias=x["bias"], h0=x["h0"])
    assert hs.shape == (0, 3, 16) and torch.equal(hT, x["h0"])
    assert (isam.linear_gru(x["gx"])[1] == 0).all()
    dgx, dh0, db = isam.linear_gru_backward(x["gx"], x["dh_seq"], states=states, bias=x["bias"], dh_T=x["dh_T"])
    assert dgx.shape == (0, 3, 32) and torch.equal(dh0, x["dh_T"]) and (db == 0).all()
    e = torch.empty((5, 0, 32), device="cuda")
    hs, hT = isam.linear_gru(e)
    assert hs.shape == (5, 0, 16) and hT.shape == (0, 16)
    db = isam.linear_gru_backward(e, e[..., :16], states=torch.empty((1, 0, 16), device="cuda"), bias=torch.zeros(32, device="cuda"))[2]
    assert (db == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [6, 60, 700, 4000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_reset_cuts_off_bad_values(T, dtype, bad):
    # a document of bad values between two good ones, and bad gradients likewise: neither the
    # states after it nor the gradients before it see them
    H, B = 40, 2
    a, b = T // 3, 2 * T // 3
    x = inputs(T, B, H, dtype, seed=T)
    r = torch.zeros((T, B), dtype=torch.bool, device="cuda")
    r[a], r[b] = True, True
    x["reset"] = r
    ref = reference(x, "linear", H)
    x["gx"][a:b, :, H:] = bad
    x["dh_seq"][a:b] = bad
    out = run(x, "linear")
    for part in (slice(0, a), slice(b, T)):
        for k in ("h_seq", "dgx"):
            check(out[k][part], (ref[k][0][part], ref[k][1][part]), f"{k} {part}")
    check(out["h_T"], ref["h_T"], "h_T")
    check(out["dh0"], ref["dh0"], "dh0")
    if bad != bad:
        assert torch.isnan(out["h_seq"][a:b].float()).all()
    # without resets a NaN stays in the state to the end
    x["reset"] = None
    if bad != bad:
        assert torch.isnan(run(x, "linear")["h_T"]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [7, 60, 700, 4000])
def test_reset_cuts_off_bad_gates(T, dtype):
    # spans of NaN gates between resets, one in every 100 steps: what follows them, and the
    # gradients of what stands before them, do not see them
    H, B = 40, 2
    x = inputs(T, B, H, dtype, seed=T)
    at = torch.arange(T)
    bad = (at % 100 >= 3) & (at % 100 < 6)
    r = (at % 100 == 3) | (at % 100 == 6)
    x["reset"] = r[:, None].expand(T, B).contiguous().cuda()
    ref = reference(x, "tanh", H)
    x["gx"][bad] = float("nan")
    out = run(x, "tanh")
    good = ~bad
    for k in ("h_seq", "dgx"):
        check(out[k][good], (ref[k][0][good], ref[k][1][good]), k)
        assert torch.isnan(out[k][bad].float()).all()
    check(out["dh0"], ref["dh0"], "dh0")
    if not bad[-1]:
        check(out["h_T"], ref["h_T"], "h_T")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [40, 700])
def test_infinite_bias(T, dtype):
    # a gate bias of either infinity is a gate shut or open; the steps past a tile's end do not see it
    H, B = 16, 2
    x = inputs(T, B, H, dtype, seed=T)
    x["bias"][1], x["bias"][2] = float("-inf"), float("inf")
    compare(x, "tanh")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_saturated_gates(dtype):
    # gates of the type's lowest and highest values and infinities: z is exactly 0 or 1
    T, B, H = 300, 2, 16
    x = inputs(T, B, H, dtype, seed=1)
    x["bias"] = None
    for i, v in enumerate((float("-inf"), float("inf"), torch.finfo(dtype).min, torch.finfo(dtype).max)):
        x["gx"][:, :, i] = v
    compare(x, "tanh")


@pytest.mark.parametrize("T,B,H", [(700, 3, 40), (5000, 1, 64), (40, 2, 16)])
def test_repeats_bit_for_bit(T, B, H):
    x = inputs(T, B, H, torch.bfloat16, seed=9, reset=0.01)
    first = run(x, "tanh")
    for _ in range(4):
        for k, v in run(x, "tanh").items():
            assert torch.equal(v, first[k]), k


@pytest.mark.parametrize("T,candidate", [(5, "tanh"), (40, "linear"), (600, "tanh")])
def test_gradient_against_differences(T, candidate):
    # central differences of the 32-bit forward pass along random directions: step 2^-6, whose third-order
    # term is below 2^-12 relative to the sums here and whose rounding is about 2^-24 * 2^6 = 2^-18
    B, H, step = 2, 24, 2.0 ** -6
    x = inputs(T, B, H, torch.float32, seed=T, reset=0.05)
    out = run(x, candidate)
    g = torch.Generator(device="cuda").manual_seed(5)

    def loss(gx, h0, bias):
        hs, hT = isam.linear_gru(gx, bias=bias, h0=h0, reset=x["reset"], candidate=candidate)
        return float((hs.double() * x["dh_seq"].double()).sum() + (hT.double() * x["dh_T"].double()).sum())

    for name, grad in (("gx", out["dgx"]), ("h0", out["dh0"]), ("bias", out["dbias"])):
        arg = {"gx": x["gx"], "h0": x["h0"], "bias": x["bias"]}
        v = torch.randn(arg[name].shape, generator=g, device="cuda")
        hi, lo = dict(arg), dict(arg)
        hi[name], lo[name] = arg[name] + step * v, arg[name] - step * v
        diff = (loss(**hi) - loss(**lo)) / (2 * step)
        size = float((grad.double() * v.double()).abs().sum())
        assert abs(diff - float((grad.double() * v.double()).sum())) <= 2.0 ** -10 * size, name


def test_other_stream():
    x = inputs(2000, 1, 64, torch.bfloat16, seed=2)
    ref = run(x, "tanh")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = run(x, "tanh")
    torch.cuda.current_stream().wait_stream(s)
    for k in ref:
        assert torch.equal(out[k], ref[k])


def test_graph_replays():
    x = inputs(2000, 1, 64, torch.bfloat16, seed=4)
    T, B, H = 2000, 1, 64
    states = torch.empty(isam.linear_gru_states_shape(T, B, H), device="cuda")
    buf = dict(h_seq=torch.empty((T, B, H), device="cuda", dtype=torch.bfloat16), h_T=torch.empty((B, H), device="cuda"))
    back = dict(dgx=torch.empty((T, B, 2 * H), device="cuda", dtype=torch.bfloat16), dh0=torch.empty((B, H), device="cuda"),
                dbias=torch.empty((2 * H,), device="cuda"))
    w1 = torch.empty(isam.linear_gru_workspace_size(T, B, H, 1), device="cuda", dtype=torch.uint8)
    w2 = torch.empty(isam.linear_gru_backward_workspace_size(T, B, H, 1), device="cuda", dtype=torch.uint8)

    def both():
        isam.linear_gru(x["gx"], bias=x["bias"], h0=x["h0"], states=states, workspace=w1, **buf)
        isam.linear_gru_backward(x["gx"], x["dh_seq"], states=states, bias=x["bias"], dh_T=x["dh_T"], workspace=w2, **back)

    both()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for i in range(3):
        x["gx"].copy_(torch.randn(x["gx"].shape, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16))
        ref = run(x, "tanh")
        g.replay()
        torch.cuda.synchronize()
        for k, v in {**buf, **back}.items():
            assert torch.equal(v, ref[k]), k


def test_long_offsets():
    # rows whose offsets pass 2^31 elements: the last steps of a long strided tensor
    T, B, H = 300, 1, 32
    stride = (1 << 31) // 256
    big = torch.empty((T * stride,), device="cuda", dtype=torch.bfloat16)
    gx = big.as_strided((T, B, 2 * H), (stride, stride, 1))
    x = inputs(T, B, H, torch.bfloat16, seed=6)
    gx.copy_(x["gx"])
    x["gx"] = gx
    compare(x, "tanh")


def test_refusals():
    T, B, H = 10, 2, 16
    x = inputs(T, B, H, torch.float32)
    ok = dict(bias=x["bias"], h0=x["h0"])
    st = torch.empty(isam.linear_gru_states_shape(T, B, H), device="cuda")
    for kw in (dict(bias=x["bias"][:5]), dict(h0=x["h0"].t()), dict(candidate="relu"), dict(reset=torch.zeros((T, B + 1), device="cuda", dtype=torch.bool)),
               dict(h_seq=torch.empty((T, B, H + 1), device="cuda")), dict(states=st[..., :3])):
        with pytest.raises(ValueError):
            isam.linear_gru(x["gx"], **{**ok, **kw})
    for kw in (dict(bias=x["bias"].double()), dict(reset=torch.zeros((T, B), device="cuda")),
               dict(h_seq=torch.empty((T, B, H), device="cuda", dtype=torch.bfloat16))):
        with pytest.raises(TypeError):
            isam.linear_gru(x["gx"], **{**ok, **kw})
    with pytest.raises(ValueError):
        isam.linear_gru(x["gx"][..., :31])
    with pytest.raises(TypeError):
        isam.linear_gru(x["gx"].half())
    with pytest.raises(ValueError):
        isam.linear_gru(x["gx"].cpu())
    with pytest.raises(isam.IsamError):      # output over input
        isam.linear_gru(x["gx"], h_seq=x["gx"][..., :H])
    with pytest.raises(isam.IsamError):      # overlapping output rows
        isam.linear_gru(x["gx"], h_seq=torch.empty((1, B, H), device="cuda").expand(T, B, H))
    with pytest.raises(isam.IsamError) as e:
        y = inputs(4000, 1, 16, torch.float32)
        isam.linear_gru(y["gx"], workspace=torch.empty(16, device="cuda", dtype=torch.uint8))
    assert e.value.status == 3
    with pytest.raises(isam.IsamError):
        isam.linear_gru_backward(x["gx"], x["dh_seq"], states=st, dgx=x["gx"])
