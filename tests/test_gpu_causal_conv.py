"""GPU parity of the causal convolution and its gradient against the definition in 64 bits.

Tolerances are formed beside the 64-bit results.  u = 2^-24: a sum of K products and a bias carries
(K + 1) u of its terms' magnitudes; silu and its slope 8 u and 2 u |p| of themselves (the exponential's
argument is rounded), twice that for the slope, whose own slope is at most 1/2; a sum over tokens at
most u for each token added.  bf16 outputs add half a step."""
import pytest
import torch

import paper_1810_09958_amd as isam

U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
pytestmark = pytest.mark.gpu


def inputs(T, B, C, K, dtype, seed=0, batch_first=False, reset=None):
    g = torch.Generator().manual_seed(seed)

    def rows(w):
        t = torch.randn((B, T, w) if batch_first else (T, B, w), generator=g).to(dtype).cuda()
        return t.transpose(0, 1) if batch_first else t

    x = dict(x=rows(C), w=torch.randn((K, C), generator=g).cuda(), bias=torch.randn(C, generator=g).cuda(),
             state=torch.randn((K - 1, B, C), generator=g).to(dtype).cuda(), reset=None, dy=rows(C),
             dstate_T=torch.randn((K - 1, B, C), generator=g).to(dtype).cuda())
    if reset is not None:
        r = (torch.rand((B, T) if batch_first else (T, B), generator=g) < reset).cuda()
        x["reset"] = r.t() if batch_first else r
    return x


def reference(x, act):
    f = {k: (v.cpu().double() if v is not None and v.is_floating_point() else v) for k, v in x.items()}
    T, B, C = f["x"].shape
    w = f["w"]
    K = w.shape[0]
    state = f["state"] if f["state"] is not None else torch.zeros((K - 1, B, C), dtype=torch.float64)
    bias = f["bias"] if f["bias"] is not None else torch.zeros(C, dtype=torch.float64)
    xs = torch.cat((state, f["x"]))
    cut = x["reset"].cpu().bool() if x["reset"] is not None else torch.zeros((T, B), dtype=torch.bool)
    # seen[t][k]: token t's tap k reads row t + k of xs, unless a reset lies after it
    seen = torch.ones((T + 1, K, B), dtype=torch.bool)      # [T]: what the state after the last token keeps
    for t in range(T + 1):
        for k in range(K):
            for s in range(max(0, t - (K - 1) + k + 1), min(t, T - 1) + 1):
                seen[t, k] &= ~cut[s]
    pre, size = bias.expand(T, B, C).clone(), bias.abs().expand(T, B, C).clone()
    for k in range(K):
        term = torch.where(seen[:T, k][..., None], xs[k:k + T] * w[k], torch.zeros((), dtype=torch.float64))
        pre, size = pre + term, size + term.abs()
    ep = (K + 1) * U * size
    if act == "silu":
        s = torch.sigmoid(pre)
        y, slope = pre * s, s * (1 + pre * (1 - s))
        ey = 1.1 * ep + y.abs() * (8 * U + 2 * U * pre.abs())
        es = 0.5 * ep + s * (1 + pre.abs()) * (16 * U + 4 * U * pre.abs())
    else:
        y, slope, ey, es = pre, torch.ones_like(pre), ep, torch.zeros_like(pre)
    zero = torch.zeros((), dtype=torch.float64)
    kept = torch.stack([torch.where(seen[T, i][..., None], xs[T + i], zero) for i in range(K - 1)]) if K > 1 else state
    out = dict(y=(y, ey), state_T=(kept, torch.zeros_like(kept)))
    dy = f["dy"] if f["dy"] is not None else torch.zeros_like(pre)
    e, ee = dy * slope, dy.abs() * es + U * (dy * slope).abs()
    dxs, edx = torch.zeros_like(xs), torch.zeros_like(xs)
    dw, edw = torch.zeros_like(w), torch.zeros_like(w)
    n = (T + B + 128) * U
    for k in range(K):
        m = seen[:T, k][..., None]
        dxs[k:k + T] += torch.where(m, w[k] * e, zero)
        edx[k:k + T] += torch.where(m, w[k].abs() * ee + (K + 1) * U * (w[k] * e).abs(), zero)
        p = torch.where(m, e * xs[k:k + T], zero)
        dw[k] = p.sum((0, 1))
        edw[k] = (torch.where(m, ee * xs[k:k + T].abs(), zero) + n * p.abs()).sum((0, 1))
    if f["dstate_T"] is not None:
        for i in range(K - 1):
            v = torch.where(seen[T, i][..., None], f["dstate_T"][i], zero)
            dxs[T + i] += v
            edx[T + i] += U * v.abs()
    edx += U * dxs.abs()
    out.update(dx=(dxs[K - 1:], edx[K - 1:]), dstate=(dxs[:K - 1], edx[:K - 1]), dw=(dw, edw),
               dbias=(e.sum((0, 1)), (ee + n * e.abs()).sum((0, 1))))
    return out


def check(got, ref, name):
    val, bound = ref
    bound = bound + HALF[got.dtype] * (val.abs() + bound) + 1e-30
    err = (got.cpu().double() - val).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / bound).max()):.2f} bounds"


def run(x, act, **kw):
    opt = {k: x[k] for k in ("bias", "state", "reset")}
    out = dict(zip(("y", "state_T"), isam.causal_conv(x["x"], x["w"], activation=act, **opt)))
    out.update(zip(("dx", "dstate", "dw", "dbias"), isam.causal_conv_backward(x["x"], x["w"], x["dy"], activation=act, dstate_T=x["dstate_T"],
                                                                             **opt, **kw)))
    torch.cuda.synchronize()
    return {k: v for k, v in out.items() if v is not None}


def compare(x, act="silu"):
    ref = reference(x, act)
    out = run(x, act)
    for k, v in out.items():
        check(v, ref[k], k)
    return out


DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])


@DTYPES
@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 6])
@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 7, 8, 9, 33, 64, 65, 300])
def test_lengths(T, K, dtype):
    compare(inputs(T, 2, 24, K, dtype, seed=T + K, reset=0.1 if T % 2 else None), "silu" if K % 2 else "none")


@DTYPES
@pytest.mark.parametrize("C", [1, 2, 3, 4, 5, 7, 8, 9, 12, 31, 64, 130, 333, 600])
def test_widths(C, dtype):
    compare(inputs(40, 3, C, 4, dtype, seed=C, reset=0.05))
    compare(inputs(2, 3, C, 3, dtype, seed=C, reset=0.3))


@DTYPES
@pytest.mark.parametrize("reset", [0.0, 0.3, 0.7, 1.0])
def test_dense_resets(reset, dtype):
    for K in (2, 4, 6):
        compare(inputs(50, 4, 10, K, dtype, seed=K, reset=reset))
        compare(inputs(3, 4, 10, K, dtype, seed=K, reset=reset))


@DTYPES
def test_long_and_batch_first(dtype):
    compare(inputs(5000, 1, 40, 4, dtype, seed=1, reset=0.002))
    compare(inputs(700, 5, 66, 3, dtype, seed=2, batch_first=True, reset=0.01), "none")


def test_optional_arguments():
    x = inputs(30, 2, 20, 4, torch.float32, seed=3)
    x["bias"] = x["state"] = x["dstate_T"] = None
    out = compare(x)
    assert "dbias" not in out
    x["dy"] = None
    x["dstate_T"] = torch.randn((3, 2, 20), device="cuda")
    compare(x)
    y, kept = isam.causal_conv(x["x"], x["w"], return_state=False)
    assert kept is None
