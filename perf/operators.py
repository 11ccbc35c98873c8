"""Performance cases of the operators of a gated recurrent language-model block.

Three operators, each with its gradient and its form for single tokens:

* ``linear_gru``: the GRU whose gates do not see the state,
  ``h_t = z_t h_{t-1} + (1 - z_t) n_t`` with ``z = sigmoid(gz + bz)`` and ``n = tanh(gn + bn)``
  (or ``gn + bn``), over sequences of any length, with resets between packed documents;
* ``gated_ffn``: ``act(x Wg^T + bg) * (x Wu^T + bu)``, both projections and the product together;
* ``norm_residual``: the norm after a block, its gate and scale, the residual sum and the norm
  before the next block: ``r' = r + s g * rms(x) w_post``, ``y = rms(r') w_pre``.

``listed()`` holds the fixed cases, ``draw(rng)`` gives more of the same ranges.  ``prepare`` makes
what a program holds before the call; ``run`` is one pass, in plain torch operations in 32 bits
(``own`` false) or by the library (``own`` true); ``work`` the bytes and operations the pass cannot
do without; ``exact`` the same results from the definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_ES = {"bf16": 2, "f32": 4}


def listed():
    return [
        # One decoding step of 32 sequences: launch latency.
        dict(name="lgru_step_bf16", op="lgru", T=1, batch=32, H=1024, dt="bf16", cand="tanh", reset=False,
             batch_first=False, train=False),
        # Reading one very long prompt: few channels, so the work has to be split along the sequence.
        dict(name="lgru_prompt_bf16", op="lgru", T=32768, batch=1, H=2048, dt="bf16", cand="tanh", reset=False,
             batch_first=False, train=False),
        # A training step of eight packed sequences stored batch first, forward and backward.
        dict(name="lgru_train_bf16", op="lgru", T=4096, batch=8, H=1024, dt="bf16", cand="tanh", reset=True,
             batch_first=True, train=True),
        # The same in fp32 with a linear candidate, at sizes that are nobody's multiple.
        dict(name="lgru_train_f32_odd", op="lgru", T=1000, batch=3, H=333, dt="f32", cand="linear", reset=True,
             batch_first=False, train=True),
        # One token through the feed-forward block: the weights are read once.
        dict(name="gffn_token_bf16", op="gffn", M=1, K=1024, F=4096, dt="bf16", act="silu", bias=False, train=False),
        # A prompt batch through a wide block: matrix-core rate.
        dict(name="gffn_prompt_bf16", op="gffn", M=8192, K=2048, F=8192, dt="bf16", act="silu", bias=False, train=False),
        # A training step over 64 steps of 32 sequences, forward and backward, with biases.
        dict(name="gffn_train_bf16", op="gffn", M=2048, K=1024, F=4096, dt="bf16", act="silu", bias=True, train=True),
        # The same in fp32, ragged.
        dict(name="gffn_train_f32_odd", op="gffn", M=500, K=511, F=771, dt="f32", act="gelu", bias=True, train=True),
        # One decoding step of 32 sequences.
        dict(name="norm_step_bf16", op="norm", R=32, D=1024, G=1, dt="bf16", post=True, backward=False),
        # Every position of a prompt batch: stream of the chip's memory.
        dict(name="norm_prompt_bf16", op="norm", R=32768, D=2048, G=1, dt="bf16", post=True, backward=False),
        # The gradient over eight sequences, each with its own gate row.
        dict(name="norm_grad_bf16", op="norm", R=8192, D=4096, G=8, dt="bf16", post=True, backward=True),
        # The gradient in fp32 with a gate for each element, ragged.
        dict(name="norm_grad_f32_odd", op="norm", R=1001, D=1537, G=1001, dt="f32", post=True, backward=True),
    ]


# ---------------------------------------------------------------------------------------
# Drawn cases
# ---------------------------------------------------------------------------------------
def _log(rng, lo, hi, step=1):
    """An integer in [lo, hi], even over its logarithm, a multiple of `step` (`lo` if that is less)."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    return max(lo, min(hi, int(v) // step * step))


def _draw_lgru(rng):
    c = dict(op="lgru", T=_log(rng, 1, 32768), batch=_log(rng, 1, 64), H=_log(rng, 32, 2048, rng.choice((1, 8, 64))),
             dt=rng.choice(("bf16", "bf16", "f32")), cand=rng.choice(("tanh", "linear")), reset=rng.random() < 0.5,
             batch_first=rng.random() < 0.5, train=rng.random() < 0.5)
    while c["T"] * c["batch"] * c["H"] > (3e7 if c["train"] or c["dt"] == "f32" else 6e7):
        key = "batch" if c["batch"] > 1 else "T"
        c[key] = c[key] // 2
    return c


def _draw_gffn(rng):
    dt = rng.choice(("bf16", "bf16", "bf16", "f32"))
    step = rng.choice((1, 8, 64))
    train = rng.random() < 0.4
    c = dict(op="gffn", M=_log(rng, 1, 8192), K=_log(rng, 64, 4096, step), F=_log(rng, 64, 8192, step), dt=dt,
             act=rng.choice(("silu", "gelu", "sigmoid")), bias=rng.random() < 0.5, train=train)
    cap = 4e9 if dt == "f32" else 2e10 if train else 1e11
    while c["M"] * c["K"] * c["F"] > cap:
        key = max(("M", "K", "F"), key=lambda n: c[n])
        c[key] = max(1, c[key] // 2 // step * step)
    return c


def _draw_norm(rng):
    D = _log(rng, 64, 8192, rng.choice((1, 8, 64)))
    parts = rng.choice((0, 1, 1, 2, 8))          # 0: a gate for each element
    R = _log(rng, 1, 32768)
    while R * D > 3e7:
        R //= 2
    if parts > 1:
        R = (R + parts - 1) // parts * parts
    return dict(op="norm", R=R, D=D, G=parts or R, dt=rng.choice(("bf16", "bf16", "f32")), post=rng.random() < 0.8,
                backward=rng.random() < 0.5)


def draw(rng):
    return rng.choice((_draw_lgru, _draw_gffn, _draw_norm))(rng)


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

    def uniform(self, shape, dt, lo, hi):
        return torch.rand(shape, generator=self.g, device=self.dev).mul_(hi - lo).add_(lo).to(_DT[dt])


_SCALE, _EPS = 0.5, 1e-6


def _inputs(c, seed):
    s, dt = _Source(seed), c["dt"]
    if c["op"] == "lgru":
        T, b, H = c["T"], c["batch"], c["H"]

        def rows(n, scale):
            if c["batch_first"]:
                return s.normal((b, T, n), dt, scale).transpose(0, 1)
            return s.normal((T, b, n), dt, scale)

        # gates that forget over a few to a few hundred steps
        x = dict(gx=rows(2 * H, 1.0), h0=s.uniform((b, H), "f32", -1.0, 1.0),
                 bias=torch.cat((s.uniform((H,), "f32", 0.0, 5.0), s.normal((H,), "f32", 0.1))))
        x["reset"] = None
        if c["reset"]:
            r = torch.rand((b, T), generator=s.g, device=s.dev) < 1 / 500
            x["reset"] = r.t() if c["batch_first"] else r.t().contiguous()
        if c["train"]:
            x["dh_seq"] = rows(H, 1.0)
            x["dh_T"] = s.normal((b, H), "f32")
        return x
    if c["op"] == "gffn":
        M, K, F = c["M"], c["K"], c["F"]
        x = dict(x=s.normal((M, K), dt), W=s.normal((2 * F, K), dt, 1 / math.sqrt(K)),
                 bias=s.normal((2 * F,), "f32", 0.1) if c["bias"] else None)
        if c["train"]:
            x["dout"] = s.normal((M, F), dt)
        return x
    R, D, G = c["R"], c["D"], c["G"]
    x = dict(x=s.normal((R, D), dt), r=s.normal((R, D), dt, 2.0), gate=s.normal((G, D), dt, 0.3),
             w_post=s.uniform((D,), "f32", 0.5, 1.5) if c["post"] else None, w_pre=s.uniform((D,), "f32", 0.5, 1.5))
    if c["backward"]:
        x["dy"] = s.normal((R, D), dt)
        x["dr_out"] = s.normal((R, D), dt)
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

    code = {"f32": isam.ISAM_F32, "bf16": isam.ISAM_BF16}[c["dt"]]
    if c["op"] == "lgru":
        T, b, H = c["T"], c["batch"], c["H"]

        def like(n):
            if c["batch_first"]:
                return torch.empty((b, T, n), device=dev, dtype=dt).transpose(0, 1)
            return torch.empty((T, b, n), device=dev, dtype=dt)

        state["fwd"] = dict(bias=x["bias"], h0=x["h0"], reset=x["reset"], candidate=c["cand"], h_seq=like(H),
                            h_T=torch.empty((b, H), device=dev),
                            workspace=room(isam.linear_gru_workspace_size(T, b, H, code)))
        if c["train"]:
            states = torch.empty(isam.linear_gru_states_shape(T, b, H), device=dev)
            state["fwd"]["states"] = states
            state["bwd"] = dict(states=states, bias=x["bias"], reset=x["reset"], candidate=c["cand"], dh_T=x["dh_T"],
                                dgx=like(2 * H), dh0=torch.empty((b, H), device=dev),
                                dbias=torch.empty((2 * H,), device=dev),
                                workspace=room(isam.linear_gru_backward_workspace_size(T, b, H, code)))
    elif c["op"] == "gffn":
        M, K, F = c["M"], c["K"], c["F"]
        state["fwd"] = dict(bias=x["bias"], activation=c["act"], out=torch.empty((M, F), device=dev, dtype=dt),
                            workspace=room(isam.gated_ffn_workspace_size(M, K, F, code)))
        if c["train"]:
            state["bwd"] = dict(bias=x["bias"], activation=c["act"], dx=torch.empty((M, K), device=dev, dtype=dt),
                                dW=torch.empty((2 * F, K), device=dev, dtype=dt),
                                dbias=torch.empty((2 * F,), device=dev) if c["bias"] else None,
                                workspace=room(isam.gated_ffn_backward_workspace_size(M, K, F, code)))
    else:
        R, D, G = c["R"], c["D"], c["G"]
        kw = dict(w_post=x["w_post"], w_pre=x["w_pre"], gate=x["gate"], scale=_SCALE, eps=_EPS)
        if c["backward"]:
            state["bwd"] = dict(kw, dr_out=x["dr_out"], dx=torch.empty((R, D), device=dev, dtype=dt),
                                dr=torch.empty((R, D), device=dev, dtype=dt),
                                dgate=torch.empty((G, D), device=dev, dtype=dt),
                                dw_post=torch.empty((D,), device=dev) if c["post"] else None,
                                dw_pre=torch.empty((D,), device=dev),
                                workspace=room(isam.norm_residual_backward_workspace_size(R, D, G, code)))
        else:
            state["fwd"] = dict(kw, r_out=torch.empty((R, D), device=dev, dtype=dt),
                                y=torch.empty((R, D), device=dev, dtype=dt))
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
        return {"lgru": _plain_lgru, "gffn": _plain_gffn, "norm": _plain_norm}[c["op"]](c, x)
    import paper_1810_09958_amd as isam
    if c["op"] == "lgru":
        out = isam.linear_gru(x["gx"], **state["fwd"])
        if c["train"]:
            out = (*out, *isam.linear_gru_backward(x["gx"], x["dh_seq"], **state["bwd"]))
        return out
    if c["op"] == "gffn":
        out = isam.gated_ffn(x["x"], x["W"], **state["fwd"])
        if c["train"]:
            return _present(out, *isam.gated_ffn_backward(x["x"], x["W"], x["dout"], **state["bwd"]))
        return out
    if c["backward"]:
        return _present(*isam.norm_residual_backward(x["x"], x["r"], x["dy"], **state["bwd"]))
    return isam.norm_residual(x["x"], x["r"], **state["fwd"])


def _plain_scan(a, b):
    """All v_t = a_t v_{t-1} + b_t with v_{-1} = 0, by doubling the span each entry covers."""
    d, T = 1, a.shape[0]
    while d < T:
        b = torch.cat((b[:d], b[d:] + a[d:] * b[:-d]))
        a = torch.cat((a[:d], a[d:] * a[:-d]))
        d *= 2
    return b


def _plain_lgru(c, x):
    H, dt = c["H"], _DT[c["dt"]]
    g = x["gx"].float() + x["bias"]
    z, n = torch.sigmoid(g[..., :H]), g[..., H:]
    if c["cand"] == "tanh":
        n = torch.tanh(n)
    a = z if x["reset"] is None else z * (~x["reset"]).float()[..., None]
    b = (1 - z) * n
    b[0] += a[0] * x["h0"]
    h = _plain_scan(a, b)
    out = (h.to(dt), h[-1])
    if not c["train"]:
        return out
    # d_t: gradient of h_t, d_t = dh_t + a_{t+1} d_{t+1}, the same scan from the end
    dh = x["dh_seq"].float()
    dh = torch.cat((dh[:-1], (dh[-1] + x["dh_T"])[None]))
    later = torch.cat((a[1:], torch.zeros_like(a[:1])))
    d = _plain_scan(later.flip(0), dh.flip(0)).flip(0)
    prev = torch.cat((x["h0"][None], h[:-1]))
    if x["reset"] is not None:
        prev = prev * (~x["reset"]).float()[..., None]
    dz = d * (prev - n) * z * (1 - z)
    dn = d * (1 - z)
    if c["cand"] == "tanh":
        dn = dn * (1 - n * n)
    dg = torch.cat((dz, dn), -1)
    return (*out, dg.to(dt), a[0] * d[0], dg.sum((0, 1)))


def _act(name, g):
    """act(g) and its derivative."""
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if name == "sigmoid" else (g * s, s * (1 + g * (1 - s)))


def _plain_gffn(c, x):
    F, dt = c["F"], _DT[c["dt"]]
    xf, W = x["x"].float(), x["W"].float()
    gu = xf @ W.t()
    if x["bias"] is not None:
        gu = gu + x["bias"]
    s, ds = _act(c["act"], gu[:, :F])
    u = gu[:, F:]
    out = (s * u).to(dt)
    if not c["train"]:
        return out
    dout = x["dout"].float()
    d = torch.cat((dout * u * ds, dout * s), 1)
    return _present(out, (d @ W).to(dt), (d.t() @ xf).to(dt), d.sum(0) if x["bias"] is not None else None)


def _plain_norm(c, x):
    R, D, G, dt = c["R"], c["D"], c["G"], _DT[c["dt"]]
    xf, r = x["x"].float(), x["r"].float()
    gate = (_SCALE * x["gate"].float()).repeat_interleave(R // G, 0) if G > 1 else _SCALE * x["gate"].float()
    q = torch.rsqrt((xf * xf).mean(1, keepdim=True) + _EPS)
    xn = xf * q if c["post"] else xf
    u = xn * x["w_post"] if c["post"] else xf
    if not c["backward"]:
        r = r + gate * u
        return r.to(dt), (r * torch.rsqrt((r * r).mean(1, keepdim=True) + _EPS) * x["w_pre"]).to(dt)
    p = torch.rsqrt((r * r).mean(1, keepdim=True) + _EPS)
    rn, dy = r * p, x["dy"].float()
    t = dy * x["w_pre"]
    dr = x["dr_out"].float() + p * (t - rn * (t * rn).mean(1, keepdim=True))
    du = gate * dr
    dgate = _SCALE * (u * dr).view(G, R // G, D).sum(1)
    dx, dw_post = du, None
    if c["post"]:
        dw_post = (du * xn).sum(0)
        t = du * x["w_post"]
        dx = q * (t - xn * (t * xn).mean(1, keepdim=True))
    return _present(dx.to(dt), dr.to(dt), dgate.to(dt), dw_post, (dy * rn).sum(0))


# ---------------------------------------------------------------------------------------
# Work, 64-bit results
# ---------------------------------------------------------------------------------------
def work(case):
    c, e = case, _ES[case["dt"]]
    if c["op"] == "lgru":
        n, ch = c["T"] * c["batch"] * c["H"], c["batch"] * c["H"]
        rows = c["T"] * c["batch"] if c["reset"] else 0
        w = dict(bytes=3 * e * n + 4 * (2 * ch + 2 * c["H"]) + rows, flops=12.0 * n)
        if c["train"]:   # the gates again and the gradient in, the gates' gradient out
            w["bytes"] += 5 * e * n + 4 * (2 * ch + 4 * c["H"]) + rows
            w["flops"] += 30.0 * n
        return w
    if c["op"] == "gffn":
        M, K, F = c["M"], c["K"], c["F"]
        b = 8 * F if c["bias"] else 0
        w = dict(bytes=e * (M * K + 2 * F * K + M * F) + b, flops=4.0 * M * K * F)
        if c["train"]:
            w["bytes"] += e * (2 * M * K + 4 * F * K + M * F) + 2 * b
            w["flops"] += 8.0 * M * K * F
        return w
    n, g, v = c["R"] * c["D"], c["G"] * c["D"], c["D"] * (2 if c["post"] else 1)
    if c["backward"]:
        return dict(bytes=e * (6 * n + 2 * g) + 8 * v, flops=30.0 * n)
    return dict(bytes=e * (4 * n + g) + 4 * v, flops=12.0 * n)


def exact(case, seed):
    c = case
    x = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in _inputs(case, seed).items()}
    return {"lgru": _exact_lgru, "gffn": _exact_gffn, "norm": _exact_norm}[c["op"]](c, x)


def _exact_lgru(c, x):
    T, H = c["T"], c["H"]
    z = 1 / (1 + torch.exp(-(x["gx"][..., :H] + x["bias"][:H])))
    n = x["gx"][..., H:] + x["bias"][H:]
    if c["cand"] == "tanh":
        n = torch.tanh(n)
    keep = torch.ones(x["gx"].shape[:2], device=z.device, dtype=torch.float64)
    if x["reset"] is not None:
        keep[x["reset"]] = 0
    kept = keep[..., None] * z
    added = n - z * n
    hs = torch.empty_like(added)
    h = x["h0"]
    for t in range(T):
        h = torch.addcmul(added[t], kept[t], h)
        hs[t] = h
    if not c["train"]:
        return hs, h.clone()
    dgx = torch.empty(x["gx"].shape, device=z.device, dtype=torch.float64)
    slope_n = (1 - z) * (1 - n * n) if c["cand"] == "tanh" else 1 - z
    d = x["dh_T"]
    for t in range(T - 1, -1, -1):
        d = d + x["dh_seq"][t]
        before = x["h0"] if t == 0 else hs[t - 1]
        dgx[t, :, :H] = d * (keep[t][:, None] * before - n[t]) * z[t] * (1 - z[t])
        dgx[t, :, H:] = d * slope_n[t]
        d = d * kept[t]
    return hs, h.clone(), dgx, d, dgx.sum(1).sum(0)


def _exact_gffn(c, x):
    F = c["F"]
    Wg, Wu = x["W"][:F], x["W"][F:]
    g, u = torch.matmul(x["x"], Wg.t().contiguous()), torch.matmul(x["x"], Wu.t().contiguous())
    if x["bias"] is not None:
        g, u = g + x["bias"][:F], u + x["bias"][F:]
    if c["act"] == "gelu":
        phi = torch.special.ndtr(g)
        s, slope = g * phi, phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    else:
        e = torch.exp(-g)
        s = 1 / (1 + e)
        slope = e / (1 + e) ** 2
        if c["act"] == "silu":
            s, slope = g * s, s + g * slope
    if not c["train"]:
        return s * u
    dg, du = x["dout"] * u * slope, x["dout"] * s
    dx = torch.matmul(dg, Wg) + torch.matmul(du, Wu)
    dW = torch.cat((torch.matmul(dg.t().contiguous(), x["x"]), torch.matmul(du.t().contiguous(), x["x"])))
    return _present(s * u, dx, dW, torch.cat((dg.sum(0), du.sum(0))) if x["bias"] is not None else None)


def _exact_norm(c, x):
    R, D, G = c["R"], c["D"], c["G"]
    gate = _SCALE * x["gate"][torch.arange(R, device=x["gate"].device) // (R // G)]
    rms_x = torch.sqrt((x["x"] ** 2).sum(1, keepdim=True) / D + _EPS)
    u = x["x"] / rms_x * x["w_post"] if c["post"] else x["x"]
    if not c["backward"]:
        r = x["r"] + gate * u
        return r, r / torch.sqrt((r ** 2).sum(1, keepdim=True) / D + _EPS) * x["w_pre"]
    r, dy = x["r"], x["dy"]
    rms_r = torch.sqrt((r ** 2).sum(1, keepdim=True) / D + _EPS)
    v = dy * x["w_pre"]
    dr = x["dr_out"] + v / rms_r - r * (v * r).sum(1, keepdim=True) / (D * rms_r ** 3)
    dgate = torch.zeros_like(x["gate"]).index_add_(0, torch.arange(R, device=r.device) // (R // G), _SCALE * u * dr)
    du = gate * dr
    dw_pre = (dy * r / rms_r).sum(0)
    if not c["post"]:
        return du, dr, dgate, dw_pre
    v = du * x["w_post"]
    dx = v / rms_x - x["x"] * (v * x["x"]).sum(1, keepdim=True) / (D * rms_x ** 3)
    return dx, dr, dgate, (du * x["x"] / rms_x).sum(0), dw_pre
