"""Performance cases of the operators of a state-space language-model block and of its decoding.

* ``linear``: a projection with its epilogue, ``act(x W^T + b) + residual``, and its gradient;
* ``causal_conv``: the short causal convolution over time before the scan, ``y_t = act(b + sum_k w_k
  x_{t-K+1+k})``, with resets between packed texts and the last inputs kept between calls, and its gradient;
* ``selective_scan``: ``h_t = exp(d_t A) h_{t-1} + d_t B_t x_t``, ``y_t = (C_t h_t + skip x_t) silu(z_t)``
  with ``d_t = softplus(dt_t + dt_bias)``, and its gradient;
* ``beam_step`` and ``beam_reorder``: one step of beam search over beams and vocabulary, and the states
  of the beams that go on.

``listed()`` holds the fixed cases, ``draw(rng)`` gives more of the same ranges.  ``prepare`` makes
what a program holds before the call; ``run`` is one pass, in plain torch operations in 32 bits
(``own`` false; 64 for the beams' scores, whose order counts) or by the library (``own`` true);
``work`` the bytes and operations the pass cannot do without; ``exact`` the same results from the
definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_ES = {"bf16": 2, "f32": 4}


def listed():
    return [
        # One token through a projection with an activation: the weights are read once.
        dict(name="lin_token_bf16", op="lin", M=1, K=1024, N=4096, dt="bf16", act="silu", bias=True, res=False, train=False),
        # A prompt batch through the projection back to the model's width, added to the residual stream.
        dict(name="lin_prompt_bf16", op="lin", M=8192, K=8192, N=2048, dt="bf16", act="none", bias=False, res=True, train=False),
        # A training step over 64 steps of 32 sequences, forward and backward, with bias and activation.
        dict(name="lin_train_bf16", op="lin", M=2048, K=1024, N=4096, dt="bf16", act="gelu", bias=True, res=False, train=True),
        # The same in fp32, ragged, with a residual.
        dict(name="lin_train_f32_odd", op="lin", M=500, K=511, N=771, dt="f32", act="silu", bias=True, res=True, train=True),
        # One decoding step of 32 sequences through the convolution: launch latency.
        dict(name="conv_step_bf16", op="conv", T=1, batch=32, C=2048, K=4, dt="bf16", act="silu", reset=False,
             batch_first=False, train=False),
        # A training step of eight packed sequences stored batch first: stream of the chip's memory.
        dict(name="conv_train_bf16", op="conv", T=4096, batch=8, C=2048, K=4, dt="bf16", act="silu", reset=True,
             batch_first=True, train=True),
        # One decoding step of 32 sequences through the scan: the states are read and written once.
        dict(name="scan_step_bf16", op="scan", T=1, batch=32, D=2048, N=16, dt="bf16", z=True, reset=False,
             batch_first=False, train=False),
        # Reading one long prompt: few channels, so the work has to be split along the sequence.
        dict(name="scan_prompt_bf16", op="scan", T=16384, batch=1, D=2048, N=16, dt="bf16", z=True, reset=False,
             batch_first=False, train=False),
        # A training step of eight packed sequences stored batch first, forward and backward.
        dict(name="scan_train_bf16", op="scan", T=2048, batch=8, D=1024, N=16, dt="bf16", z=True, reset=True,
             batch_first=True, train=True),
        # The same in fp32 without the gate, at sizes that are nobody's multiple.
        dict(name="scan_train_f32_odd", op="scan", T=500, batch=3, D=333, N=13, dt="f32", z=False, reset=True,
             batch_first=False, train=True),
        # One text, four beams over the example model's vocabulary: launch latency.
        dict(name="beam_small_f32", op="beam", batch=1, beams=4, width=4, V=256, dt="f32", done=False, layers=2, H=512),
        # 32 texts of eight beams over a large vocabulary, some of them finished, and their states.
        dict(name="beam_batch_f32", op="beam", batch=32, beams=8, width=8, V=32000, dt="f32", done=True, layers=8, H=2048),
    ]


# ---------------------------------------------------------------------------------------
# Drawn cases
# ---------------------------------------------------------------------------------------
def _log(rng, lo, hi, step=1):
    """An integer in [lo, hi], even over its logarithm, a multiple of `step` (`lo` if that is less)."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    return max(lo, min(hi, int(v) // step * step))


def _draw_lin(rng):
    dt = rng.choice(("bf16", "bf16", "bf16", "f32"))
    step = rng.choice((1, 8, 64))
    train = rng.random() < 0.4
    c = dict(op="lin", M=_log(rng, 1, 8192), K=_log(rng, 64, 8192, step), N=_log(rng, 64, 8192, step), dt=dt,
             act=rng.choice(("none", "sigmoid", "silu", "gelu")), bias=rng.random() < 0.5, res=rng.random() < 0.5, train=train)
    cap = 4e9 if dt == "f32" else 2e10 if train else 1.2e11
    while c["M"] * c["K"] * c["N"] > cap:
        key = max(("M", "K", "N"), key=lambda n: c[n])
        c[key] = max(1, c[key] // 2 // step * step)
    return c


def _shrink(c, size, cap):
    while size(c) > cap:
        key = "batch" if c["batch"] > 1 else "T"
        c[key] = c[key] // 2
    return c


def _draw_conv(rng):
    c = dict(op="conv", T=_log(rng, 1, 32768), batch=_log(rng, 1, 64), C=_log(rng, 32, 4096, rng.choice((1, 8, 64))),
             K=rng.choice((2, 3, 4, 4, 5)), dt=rng.choice(("bf16", "bf16", "f32")), act=rng.choice(("none", "silu")),
             reset=rng.random() < 0.5, batch_first=rng.random() < 0.5, train=rng.random() < 0.5)
    return _shrink(c, lambda c: c["T"] * c["batch"] * c["C"], 6e7)


def _draw_scan(rng):
    c = dict(op="scan", T=_log(rng, 1, 16384), batch=_log(rng, 1, 32), D=_log(rng, 32, 4096, rng.choice((1, 8, 64))),
             N=rng.choice((4, 7, 8, 13, 16, 16, 16, 24, 32, 64)), dt=rng.choice(("bf16", "bf16", "f32")),
             z=rng.random() < 0.7, reset=rng.random() < 0.5, batch_first=rng.random() < 0.5, train=rng.random() < 0.5)
    return _shrink(c, lambda c: c["T"] * c["batch"] * c["D"] * c["N"], 2e8 if c["train"] else 5e8)


def _draw_beam(rng):
    c = dict(op="beam", batch=_log(rng, 1, 64), beams=_log(rng, 1, 16), width=0, V=_log(rng, 64, 131072),
             dt=rng.choice(("bf16", "f32")), done=rng.random() < 0.5, layers=rng.choice((1, 2, 8)),
             H=_log(rng, 64, 2048, rng.choice((1, 8))))
    c["width"] = c["beams"] if rng.random() < 0.7 else _log(rng, 1, 16)
    while c["batch"] * c["beams"] * c["V"] > 8e6:
        c["batch" if c["batch"] > 1 else "V"] //= 2
    return c


def draw(rng):
    return rng.choice((_draw_lin, _draw_conv, _draw_scan, _draw_scan, _draw_beam))(rng)


# ---------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------
class _Source:
    def __init__(self, seed):
        self.dev = torch.device("cuda")
        self.g = torch.Generator(device=self.dev)
        self.g.manual_seed(int(seed))

    def normal(self, shape, dt, scale=1.0):
        return torch.randn(shape, generator=self.g, device=self.dev).mul_(scale).to(_DT[dt])

    def uniform(self, shape, lo, hi):
        return torch.rand(shape, generator=self.g, device=self.dev).mul_(hi - lo).add_(lo)

    def rows(self, c, width, dt):
        """[T][batch][width] in the case's order of storage."""
        if c["batch_first"]:
            return self.normal((c["batch"], c["T"], width), dt).transpose(0, 1)
        return self.normal((c["T"], c["batch"], width), dt)

    def resets(self, c):
        if not c["reset"]:
            return None
        r = torch.rand((c["batch"], c["T"]), generator=self.g, device=self.dev) < 1 / 500
        return r.t() if c["batch_first"] else r.t().contiguous()


_END = 2     # the token that ends a text


def _inputs(c, seed):
    s, dt = _Source(seed), c["dt"]
    if c["op"] == "lin":
        M, K, N = c["M"], c["K"], c["N"]
        x = dict(x=s.normal((M, K), dt), W=s.normal((N, K), dt, 1 / math.sqrt(K)),
                 bias=s.normal((N,), "f32", 0.1) if c["bias"] else None, res=s.normal((M, N), dt) if c["res"] else None)
        if c["train"]:
            x["dout"] = s.normal((M, N), dt)
        return x
    if c["op"] == "conv":
        K, C, b = c["K"], c["C"], c["batch"]
        x = dict(x=s.rows(c, C, dt), w=s.normal((K, C), "f32", 1 / math.sqrt(K)), bias=s.normal((C,), "f32", 0.1),
                 state=s.normal((K - 1, b, C), dt), reset=s.resets(c))
        if c["train"]:
            x["dy"] = s.rows(c, C, dt)
            x["dstate_T"] = s.normal((K - 1, b, C), dt)
        return x
    if c["op"] == "scan":
        b, D, N = c["batch"], c["D"], c["N"]
        # x and z are halves of one projection, B and C of another; steps of 0.001 to 0.1, states that
        # live from a few steps to a few thousand
        xz = s.rows(c, 2 * D if c["z"] else D, dt)
        bc = s.rows(c, 2 * N, dt)
        step = torch.exp(s.uniform((D,), math.log(0.001), math.log(0.1)))
        x = dict(x=xz[..., :D], z=xz[..., D:] if c["z"] else None, dt=s.rows(c, D, dt), B=bc[..., :N], C=bc[..., N:],
                 A=-s.uniform((D, N), 0.5, 1.5) * torch.arange(1, N + 1, device=s.dev), skip=s.uniform((D,), 0.5, 1.5),
                 dt_bias=torch.log(torch.expm1(step)), h0=s.normal((b, D, N), "f32"), reset=s.resets(c))
        if c["train"]:
            x["dy"] = s.rows(c, D, dt)
            x["dh_T"] = s.normal((b, D, N), "f32")
        return x
    b, n = c["batch"], c["beams"]
    x = dict(logits=s.normal((b, n, c["V"]), dt, 3.0), scores=s.uniform((b, n), -20.0, -5.0),
             state=s.normal((c["layers"], b * n, c["H"]), "f32"), finished=None)
    if c["done"]:
        x["finished"] = torch.rand((b, n), generator=s.g, device=s.dev) < 0.2
    return x


def prepare(case, seed):
    c, x = case, _inputs(case, seed)
    state = dict(case=c, x=x)
    if not own:
        return state
    import paper_1810_09958_amd as isam
    dev, dt = torch.device("cuda"), _DT[c["dt"]]

    def room(nbytes):
        return torch.empty(max(nbytes, 1), device=dev, dtype=torch.uint8)

    def f32(*shape):
        return torch.empty(shape, device=dev)

    def like(width):
        if c["batch_first"]:
            return torch.empty((c["batch"], c["T"], width), device=dev, dtype=dt).transpose(0, 1)
        return torch.empty((c["T"], c["batch"], width), device=dev, dtype=dt)

    code = {"f32": isam.ISAM_F32, "bf16": isam.ISAM_BF16}[c["dt"]]
    if c["op"] == "lin":
        M, K, N = c["M"], c["K"], c["N"]
        state["fwd"] = dict(bias=x["bias"], activation=c["act"], residual=x["res"], out=torch.empty((M, N), device=dev, dtype=dt),
                            workspace=room(isam.linear_workspace_size(M, K, N, code)))
        if c["train"]:
            state["bwd"] = dict(bias=x["bias"], activation=c["act"], dx=torch.empty((M, K), device=dev, dtype=dt),
                                dW=torch.empty((N, K), device=dev, dtype=dt), dbias=f32(N) if c["bias"] else None,
                                workspace=room(isam.linear_backward_workspace_size(M, K, N, code)))
    elif c["op"] == "conv":
        T, b, C, K = c["T"], c["batch"], c["C"], c["K"]
        state["fwd"] = dict(bias=x["bias"], state=x["state"], reset=x["reset"], activation=c["act"], y=like(C),
                            state_T=torch.empty((K - 1, b, C), device=dev, dtype=dt))
        if c["train"]:
            state["bwd"] = dict(bias=x["bias"], state=x["state"], reset=x["reset"], activation=c["act"], dstate_T=x["dstate_T"],
                                dx=like(C), dstate=torch.empty((K - 1, b, C), device=dev, dtype=dt), dw=f32(K, C), dbias=f32(C),
                                workspace=room(isam.causal_conv_backward_workspace_size(T, b, C, K, code)))
    elif c["op"] == "scan":
        T, b, D, N = c["T"], c["batch"], c["D"], c["N"]
        par = dict(skip=x["skip"], z=x["z"], dt_bias=x["dt_bias"], reset=x["reset"])
        state["fwd"] = dict(par, h0=x["h0"], y=like(D), h_T=f32(b, D, N),
                            workspace=room(isam.selective_scan_workspace_size(T, b, D, N, code)))
        if c["train"]:
            states = f32(*isam.selective_scan_states_shape(T, b, D, N))
            state["fwd"]["states"] = states
            state["bwd"] = dict(par, states=states, dh_T=x["dh_T"], dx=like(D), ddt=like(D), dA=f32(D, N), dB=like(N), dC=like(N),
                                dskip=f32(D), dz=like(D) if c["z"] else None, ddt_bias=f32(D), dh0=f32(b, D, N),
                                workspace=room(isam.selective_scan_backward_workspace_size(T, b, D, N, code)))
    else:
        b, n, w = c["batch"], c["beams"], c["width"]
        state["step"] = dict(width=w, finished=x["finished"], end=_END, scores_out=f32(b, w),
                             parent=torch.empty((b, w), device=dev, dtype=torch.int32),
                             token=torch.empty((b, w), device=dev, dtype=torch.int32),
                             finished_out=torch.empty((b, w), device=dev, dtype=torch.bool),
                             workspace=room(isam.beam_step_workspace_size(b, n, c["V"], w, code)))
        state["out"] = f32(c["layers"], b * w, c["H"])
    return state


# ---------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------
def _present(*outputs):
    """The outputs that the case has (no bias, no gradient of one)."""
    return tuple(t for t in outputs if t is not None)


def run(state):
    c, x = state["case"], state["x"]
    if not own:
        return {"lin": _plain_lin, "conv": _plain_conv, "scan": _plain_selective, "beam": _plain_beam}[c["op"]](c, x)
    import paper_1810_09958_amd as isam
    if c["op"] == "lin":
        out = isam.linear(x["x"], x["W"], **state["fwd"])
        if c["train"]:
            return _present(out, *isam.linear_backward(x["x"], x["W"], x["dout"], **state["bwd"]))
        return out
    if c["op"] == "conv":
        out = isam.causal_conv(x["x"], x["w"], **state["fwd"])
        if c["train"]:
            out = (*out, *isam.causal_conv_backward(x["x"], x["w"], x["dy"], **state["bwd"]))
        return out
    if c["op"] == "scan":
        seq = (x["x"], x["dt"], x["A"], x["B"], x["C"])
        out = isam.selective_scan(*seq, **state["fwd"])
        if c["train"]:
            out = _present(*out, *isam.selective_scan_backward(*seq, x["dy"], **state["bwd"]))
        return out
    scores, parent, token, finished = isam.beam_step(x["logits"], x["scores"], **state["step"])
    return scores, parent, token, finished, isam.beam_reorder(x["state"], parent, dim=1, out=state["out"])


def _act(name, g):
    """act(g) and its derivative."""
    if name == "none":
        return g, torch.ones_like(g)
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if name == "sigmoid" else (g * s, s * (1 + g * (1 - s)))


def _plain_lin(c, x):
    dt = _DT[c["dt"]]
    xf, W = x["x"].float(), x["W"].float()
    g = xf @ W.t()
    if x["bias"] is not None:
        g = g + x["bias"]
    s, ds = _act(c["act"], g)
    out = (s if x["res"] is None else s + x["res"].float()).to(dt)
    if not c["train"]:
        return out
    d = x["dout"].float() * ds
    return _present(out, (d @ W).to(dt), (d.t() @ xf).to(dt), d.sum(0) if x["bias"] is not None else None)


def _plain_conv(c, x):
    T, b, C, K, dt = c["T"], c["batch"], c["C"], c["K"], _DT[c["dt"]]
    xs = torch.cat((x["state"], x["x"])).float()           # step t at row t + K - 1
    # steps since the last reset: tap k of step t sees step t - j (j = K - 1 - k) if no reset lies after it
    since = torch.full((T, b), K, device=xs.device)
    if x["reset"] is not None:
        at = torch.where(x["reset"], torch.arange(T, device=xs.device)[:, None], -K).cummax(0).values
        since = torch.arange(T, device=xs.device)[:, None] - at
    seen = [(since >= j)[..., None] for j in range(K)]
    pre = x["bias"].expand(T, b, C)
    for k in range(K):
        pre = pre + x["w"][k] * (xs[k:k + T] * seen[K - 1 - k])
    y, slope = _act(c["act"], pre)
    rest = since[-1] if T else None
    kept = [xs[T + i] * (rest >= K - 2 - i)[..., None] for i in range(K - 1)]
    out = (y.to(dt), torch.stack(kept).to(dt))
    if not c["train"]:
        return out
    d = x["dy"].float() * slope
    dxs = torch.zeros_like(xs)
    dw = []
    for k in range(K):
        dk = d * seen[K - 1 - k]
        dw.append((dk * xs[k:k + T]).sum((0, 1)))
        dxs[k:k + T] += x["w"][k] * dk
    for i in range(K - 1):
        dxs[T + i] += x["dstate_T"][i].float() * (rest >= K - 2 - i)[..., None]
    return (*out, dxs[K - 1:].to(dt), dxs[:K - 1].to(dt), torch.stack(dw), d.sum((0, 1)))


def _plain_scan(a, b):
    """All v_t = a_t v_{t-1} + b_t with v_{-1} = 0, by doubling the span each entry covers."""
    d, T = 1, a.shape[0]
    while d < T:
        b = torch.cat((b[:d], b[d:] + a[d:] * b[:-d]))
        a = torch.cat((a[:d], a[d:] * a[:-d]))
        d *= 2
    return b


def _softplus(v):
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))


def _plain_selective(c, x):
    dt = _DT[c["dt"]]
    xf, Bf, Cf = x["x"].float(), x["B"].float()[:, :, None], x["C"].float()[:, :, None]
    raw = x["dt"].float() + x["dt_bias"]
    step = _softplus(raw)
    a = torch.exp(step[..., None] * x["A"])                # [T][batch][D][N]
    if x["reset"] is not None:
        a = a * (~x["reset"]).float()[..., None, None]
    b = (step * xf)[..., None] * Bf
    b[0] += a[0] * x["h0"]
    h = _plain_scan(a, b)
    v = (h * Cf).sum(-1) + x["skip"] * xf
    gate = slope = None
    if x["z"] is not None:
        gate, slope = _act("silu", x["z"].float())
    out = ((v if gate is None else v * gate).to(dt), h[-1].clone())
    if not c["train"]:
        return out
    dy = x["dy"].float()
    dv, dz = (dy, None) if gate is None else (dy * gate, (dy * v * slope).to(dt))
    # g_t: gradient of h_t, g_t = C_t dv_t + a_{t+1} g_{t+1}, the same scan from the end
    g = dv[..., None] * Cf
    g[-1] += x["dh_T"]
    later = torch.cat((a[1:], torch.zeros_like(a[:1])))
    g = _plain_scan(later.flip(0), g.flip(0)).flip(0)
    del later
    dC = (h * dv[..., None]).sum(2)
    prev = torch.cat((x["h0"][None], h[:-1]))
    del h, b
    dB = (g * (step * xf)[..., None]).sum(2)
    gB = (g * Bf).sum(-1)
    q = g * a * prev
    del prev
    dstep = (q * x["A"]).sum(-1) + gB * xf
    ddt = dstep * torch.sigmoid(raw)
    return _present(*out, (x["skip"] * dv + step * gB).to(dt), ddt.to(dt), (q * step[..., None]).sum((0, 1)), dB.to(dt), dC.to(dt),
                    (dv * xf).sum((0, 1)), dz, ddt.sum((0, 1)), a[0] * g[0])


def _plain_beam(c, x):
    b, n, V, w = c["batch"], c["beams"], c["V"], c["width"]
    logits = x["logits"].double()
    top = logits.max(-1, keepdim=True).values
    logp = logits - (top + torch.log(torch.exp(logits - top).sum(-1, keepdim=True)))
    if x["finished"] is not None:                            # a finished beam goes on unchanged, by the end token
        only = torch.full((V,), -math.inf, device=logits.device, dtype=torch.float64)
        only[_END] = 0
        logp = torch.where(x["finished"][..., None], only, logp)
    total = (x["scores"].double()[..., None] + logp).view(b, n * V)
    best, at = total.sort(dim=1, descending=True, stable=True)
    best, at = best[:, :w], at[:, :w]
    parent, token = at // V, at % V
    finished = token == _END
    if x["finished"] is not None:
        finished = finished | x["finished"].gather(1, parent)
    rows = (parent + torch.arange(b, device=at.device)[:, None] * n).reshape(-1)
    return best.float(), parent.int(), token.int(), finished, x["state"][:, rows]


# ---------------------------------------------------------------------------------------
# Work, 64-bit results
# ---------------------------------------------------------------------------------------
def work(case):
    c, e = case, _ES[case["dt"]]
    if c["op"] == "lin":
        M, K, N = c["M"], c["K"], c["N"]
        b = 4 * N if c["bias"] else 0
        w = dict(bytes=e * (M * K + N * K + M * N * (2 if c["res"] else 1)) + b, flops=2.0 * M * K * N)
        if c["train"]:
            w["bytes"] += e * (2 * M * K + 2 * N * K + M * N) + 2 * b
            w["flops"] += 4.0 * M * K * N
        return w
    if c["op"] == "conv":
        n, s, K = c["T"] * c["batch"] * c["C"], (c["K"] - 1) * c["batch"] * c["C"], c["K"]
        rows, par = (c["T"] * c["batch"] if c["reset"] else 0), 4 * (K + 1) * c["C"]
        w = dict(bytes=e * (2 * n + 2 * s) + par + rows, flops=2.0 * K * n)
        if c["train"]:
            w["bytes"] += e * (3 * n + 3 * s) + 2 * par + rows
            w["flops"] += 6.0 * K * n
        return w
    if c["op"] == "scan":
        n, m, h = c["T"] * c["batch"] * c["D"], c["T"] * c["batch"] * c["N"], c["batch"] * c["D"] * c["N"]
        z, par, rows = (1 if c["z"] else 0), 4 * c["D"] * (c["N"] + 2), (c["T"] * c["batch"] if c["reset"] else 0)
        # exp, two products and two multiplications with an addition for each value of the state
        w = dict(bytes=e * ((3 + z) * n + 2 * m) + 8 * h + par + rows, flops=7.0 * n * c["N"])
        if c["train"]:
            w["bytes"] += e * ((5 + 2 * z) * n + 4 * m) + 8 * h + 2 * par + rows
            w["flops"] += 18.0 * n * c["N"]
        return w
    rows, out = c["batch"] * c["beams"], c["batch"] * c["width"]
    return dict(bytes=e * rows * c["V"] + 5 * rows + 13 * out + 8 * out * c["layers"] * c["H"], flops=4.0 * rows * c["V"])


def exact(case, seed):
    c = case
    x = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in _inputs(case, seed).items()}
    return {"lin": _exact_lin, "conv": _exact_conv, "scan": _exact_selective, "beam": _exact_beam}[c["op"]](c, x)


def _exact_act(name, g):
    if name == "none":
        return g, torch.ones((), device=g.device, dtype=torch.float64)
    if name == "gelu":
        phi = torch.special.ndtr(g)
        return g * phi, phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    e = torch.exp(-g)
    s, slope = 1 / (1 + e), e / (1 + e) ** 2
    return (s, slope) if name == "sigmoid" else (g * s, s + g * slope)


def _exact_lin(c, x):
    g = torch.matmul(x["x"], x["W"].t().contiguous())
    if x["bias"] is not None:
        g += x["bias"]
    out, slope = _exact_act(c["act"], g)
    if x["res"] is not None:
        out = out + x["res"]
    if not c["train"]:
        return out
    d = x["dout"] * slope
    return _present(out, torch.matmul(d, x["W"]), torch.matmul(d.t().contiguous(), x["x"]), d.sum(0) if x["bias"] is not None else None)


def _exact_conv(c, x):
    # step by step, with the window of inputs that a step still sees
    T, K, w = c["T"], c["K"], x["w"]
    window = list(x["state"])
    pre = torch.empty(x["x"].shape, device=w.device, dtype=torch.float64)
    seen = []
    for t in range(T):
        window.append(x["x"][t])
        if x["reset"] is not None:
            keep = (~x["reset"][t])[:, None].double()
            window = [v * keep for v in window[:-1]] + window[-1:]
        pre[t] = x["bias"] + sum(w[k] * window[k] for k in range(K))
        if c["train"]:
            seen.append(torch.stack(window))
        window = window[1:]
    y, slope = _exact_act(c["act"], pre)
    out = (y, torch.stack(window))
    if not c["train"]:
        return out
    d = x["dy"] * slope
    dx = torch.empty_like(pre)
    dw = torch.zeros_like(w)
    back = list(x["dstate_T"])                        # gradients of the window after step t
    for t in range(T - 1, -1, -1):
        full = [0 * d[t]] + back
        full = [full[k] + w[k] * d[t] for k in range(K)]
        dw += (seen[t] * d[t]).sum(1)
        dx[t] = full[K - 1]
        back = full[:-1]
        if x["reset"] is not None:
            keep = (~x["reset"][t])[:, None].double()
            back = [v * keep for v in back]
    return (*out, dx, torch.stack(back), dw, d.sum(1).sum(0))


def _exact_selective(c, x):
    T, A = c["T"], x["A"]
    raw = x["dt"] + x["dt_bias"]
    step = torch.nn.functional.softplus(raw, threshold=100)
    keep = torch.ones(x["dt"].shape[:2], device=A.device, dtype=torch.float64)
    if x["reset"] is not None:
        keep[x["reset"]] = 0
    h, hs = x["h0"], []
    v = x["skip"] * x["x"]
    for t in range(T):
        h = torch.exp(step[t][..., None] * A) * (h * keep[t][:, None, None]) + (step[t] * x["x"][t])[..., None] * x["B"][t][:, None]
        v[t] += (h * x["C"][t][:, None]).sum(-1)
        if c["train"]:
            hs.append(h)
    s, slope = _exact_act("silu", x["z"]) if x["z"] is not None else (None, None)
    out = (v if s is None else v * s, h.clone())
    if not c["train"]:
        return out
    dv = x["dy"] if s is None else x["dy"] * s
    dz = None if s is None else x["dy"] * v * slope
    dx, ddt = x["skip"] * dv, torch.empty_like(step)
    dA, dB, dC = torch.zeros_like(A), torch.empty_like(x["B"]), torch.empty_like(x["C"])
    g = x["dh_T"]
    for t in range(T - 1, -1, -1):
        before = (x["h0"] if t == 0 else hs[t - 1]) * keep[t][:, None, None]
        g = g + dv[t][..., None] * x["C"][t][:, None]
        dC[t] = (hs[t] * dv[t][..., None]).sum(1)
        dB[t] = (g * (step[t] * x["x"][t])[..., None]).sum(1)
        pulled = (g * x["B"][t][:, None]).sum(-1)
        dx[t] += step[t] * pulled
        g = g * torch.exp(step[t][..., None] * A)
        ddt[t] = ((g * before * A).sum(-1) + pulled * x["x"][t]) / (1 + torch.exp(-raw[t]))
        dA += (g * before * step[t][..., None]).sum(0)
        g = g * keep[t][:, None, None]
        hs[t] = None
    return _present(*out, dx, ddt, dA, dB, dC, (dv * x["x"]).sum(1).sum(0), dz, ddt.sum(1).sum(0), g)


def _exact_beam(c, x):
    b, n, V, w = c["batch"], c["beams"], c["V"], c["width"]
    total = x["scores"][..., None] + x["logits"] - torch.logsumexp(x["logits"], -1, keepdim=True)
    if x["finished"] is not None:
        total[x["finished"]] = -math.inf
        total[..., _END] = torch.where(x["finished"], x["scores"], total[..., _END])
    flat = total.reshape(b, n * V)
    taken = torch.zeros_like(flat, dtype=torch.bool)
    scores, parents, tokens = [], [], []
    for _ in range(w):                                # the best, lowest index first, one by one
        best = flat.masked_fill(taken, -math.inf).max(1, keepdim=True).values
        at = ((flat == best) & ~taken).double().argmax(1, keepdim=True)
        scores.append(best)
        parents.append(at // V)
        tokens.append(at % V)
        taken.scatter_(1, at, True)
    score, parent, token = (torch.cat(v, 1) for v in (scores, parents, tokens))
    done = token == _END
    if x["finished"] is not None:
        done |= x["finished"].gather(1, parent)
    state = x["state"].view(c["layers"], b, n, c["H"])
    state = torch.stack([state[:, i, parent[i]] for i in range(b)], 1).reshape(c["layers"], b * w, c["H"])
    return score, parent.int(), token.int(), done, state
