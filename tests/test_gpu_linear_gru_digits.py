"""The linear GRU's digits where its values are small, against the recurrence in 64 bits.

u = 2^-24.  A gate value or candidate carries a relative error of at most 32 u, however small it is (a sum
of input and bias that cancels is exact), so a step adds at most 32 u (|z h| + 2 |(1-z) n|) to what z leaves
of the error before it, and a gradient's factors 32 u each.  bf16 outputs add half a unit in their last place."""
import pytest
import torch

import paper_1810_09958_amd as isam

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STEP = 32 * U
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}


def reference(gx, bias, dh_seq):
    """tanh candidate, zero h0 and dh_T, no resets: name -> (64-bit value, bound of the error)."""
    g = gx.double() + bias.double()
    T, B, H2 = g.shape
    H = H2 // 2
    z, w, n = torch.sigmoid(g[..., :H]), torch.sigmoid(-g[..., :H]), torch.tanh(g[..., H:])
    h = eh = torch.zeros((B, H), device=g.device, dtype=torch.float64)
    hs, ehs = [h], [eh]
    for t in range(T):
        h, eh = z[t] * h + w[t] * n[t], z[t] * eh + STEP * ((z[t] * h).abs() + 2 * (w[t] * n[t]).abs())
        hs.append(h)
        ehs.append(eh)
    hs, ehs = torch.stack(hs), torch.stack(ehs)
    e, ee = torch.zeros_like(h), torch.zeros_like(h)
    dg, edg = torch.zeros_like(g), torch.zeros_like(g)
    for t in range(T - 1, -1, -1):
        d = dh_seq[t].double() + e
        ed, diff, s = ee + U * d.abs(), hs[t] - n[t], z[t] * w[t]
        dg[t, :, :H] = d * diff * s
        edg[t, :, :H] = s * (ed * diff.abs() + d.abs() * (ehs[t] + 4 * STEP * (hs[t].abs() + n[t].abs())))
        dg[t, :, H:] = d * w[t] * (1 - n[t] ** 2)
        edg[t, :, H:] = w[t] * (ed + d.abs() * 3 * STEP)
        e, ee = z[t] * d, z[t] * (ed + STEP * d.abs())
    return dict(h_seq=(hs[1:], ehs[1:]), h_T=(h, eh), dgx=(dg, edg), dh0=(e, ee),
                dbias=(dg.sum((0, 1)), edg.sum((0, 1)) + 64 * U * dg.abs().sum((0, 1))))


def check(gx, bias, seed):
    T, B, H2 = gx.shape
    g = torch.Generator().manual_seed(seed)
    dh = torch.randn((T, B, H2 // 2), generator=g).to(gx.dtype).cuda()
    states = torch.empty(isam.linear_gru_states_shape(T, B, H2 // 2), device="cuda")
    out = {}
    out["h_seq"], out["h_T"] = isam.linear_gru(gx, bias=bias, states=states)
    out["dgx"], out["dh0"], out["dbias"] = isam.linear_gru_backward(gx, dh, states=states, bias=bias)
    for k, (val, bound) in reference(gx, bias, dh).items():
        err = (out[k].double() - val).abs()
        bound = bound + HALF[out[k].dtype] * val.abs() + 1e-40
        assert (err <= bound).all(), f"{k}: worst {float((err / bound).max()):.2f} bounds"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [3, 40, 300])
@pytest.mark.parametrize("size", [1.0, 0.3, 0.1, 1e-3, 1e-5, 1e-6, 1e-20])
def test_small_candidates(size, T, dtype):
    H = 40
    g = torch.Generator().manual_seed(T)
    gx = torch.randn((T, 2, 2 * H), generator=g)
    gx[..., H:] *= size
    bias = torch.cat((torch.rand(H, generator=g) * 6 - 1, torch.randn(H, generator=g) * size))
    check(gx.to(dtype).cuda(), bias.cuda(), T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [3, 40, 300])
@pytest.mark.parametrize("rest", [0.1, 1e-3, 1e-5])
def test_bias_that_cancels(rest, T, dtype):
    # inputs of -3 to 3 in the candidate, and of up to 1000 in the gate, that their bias takes back but for `rest`
    # (2^-20 and more of each, so the difference is exact in 32 bits)
    H = 40
    g = torch.Generator().manual_seed(T)
    row = torch.cat((torch.randint(-1000, 1001, (H,), generator=g).float(), torch.randint(-24, 25, (H,), generator=g) / 8))
    gx = row.to(torch.bfloat16).to(dtype).expand(T, 2, 2 * H).contiguous().cuda()
    off = torch.cat((torch.randn(H, generator=g), rest * torch.randn(H, generator=g)))
    bias = (off - row.to(torch.bfloat16).float()).cuda()
    check(gx, bias, T)


def _near_steps(T, B, H, dtype, seed):
    from tests.test_gpu_linear_gru import compare, inputs
    compare(inputs(T, B, H, dtype, seed=seed, reset=0.01), "tanh")


# A row's last piece of four channels may begin inside the piece before it (two channels of it at 6 and 70, across
# two workgroups' channels at 66 and 130); time around one backward tile.
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,H", [(300, 4), (300, 5), (300, 6), (300, 30), (300, 66), (300, 70), (300, 130), (20, 66), (127, 66),
                                 (128, 66), (129, 66), (127, 40), (128, 40), (129, 40), (384, 40), (385, 40)])
def test_overlapping_pieces_and_tile_ends(T, H, dtype):
    _near_steps(T, 2, H, dtype, T + H)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_step_has_no_stride(dtype):
    # one step cut out of a tensor whose steps lie 2^29 values apart: forward and backward
    from tests.test_gpu_linear_gru import check as check_bounds, inputs, reference as full
    B, H, far = 3, 24, 1 << 29
    x = inputs(1, B, H, dtype, seed=1, reset=0.5)
    ref = full(x, "tanh", H)

    def apart(w):
        return torch.zeros((B, w), device="cuda", dtype=dtype).as_strided((1, B, w), (far, w, 1))

    gx, dh, h, dgx = apart(2 * H), apart(H), apart(H), apart(2 * H)
    gx.copy_(x["gx"])
    dh.copy_(x["dh_seq"])
    reset = x["reset"].contiguous().as_strided((1, B), (1 << 30, 1))
    states = torch.empty(isam.linear_gru_states_shape(1, B, H), device="cuda")
    _, h_T = isam.linear_gru(gx, bias=x["bias"], h0=x["h0"], reset=reset, h_seq=h, states=states)
    _, dh0, db = isam.linear_gru_backward(gx, dh, states=states, bias=x["bias"], reset=reset, dh_T=x["dh_T"], dgx=dgx)
    for k, v in (("h_seq", h), ("h_T", h_T), ("dgx", dgx), ("dh0", dh0), ("dbias", db)):
        check_bounds(v, ref[k], k)


def test_few_steps_far_apart():
    # eight steps 2^25 values apart: 32 of them would pass 2^31 bytes
    from tests.test_gpu_linear_gru import check as check_bounds, inputs, reference as full
    T, B, H, far = 8, 2, 24, 1 << 25
    x = inputs(T, B, H, torch.bfloat16, seed=2, train=False)
    ref = full(x, "tanh", H)
    gx = torch.empty(((T - 1) * far + 2 * B * H,), device="cuda", dtype=torch.bfloat16).as_strided((T, B, 2 * H), (far, 2 * H, 1))
    gx.copy_(x["gx"])
    h, h_T = isam.linear_gru(gx, bias=x["bias"], h0=x["h0"])
    check_bounds(h, ref["h_seq"], "h_seq")
    check_bounds(h_T, ref["h_T"], "h_T")
    with pytest.raises(isam.IsamError) as e:       # a gradient forms tiles of time
        isam.linear_gru_backward(gx, None, states=torch.empty((1, B, H), device="cuda"), bias=x["bias"])
    assert e.value.status == 2
