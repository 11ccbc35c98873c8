"""A small language model of state-space blocks, trained and decoded with the library's operators.

    r_0 = E[token],                                   y = norm(r)            before each half of a layer
    x z = linear(y, Wi)                               x = causal_conv(x)
    s B C = linear(x, Wx),  dt = linear(s, Wdt)       h = selective_scan(x, dt, A, B, C, z)
    r = linear(h, Wo, residual=r)                     (a layer's first half)
    r = linear(linear(y, W1, gelu), W2, residual=r)   (its second half)
    logits = norm(r) E^T

Activations are rows [T * batch][width], time first, so one call covers a prompt, a training step or (T = 1)
one token of every sequence.  ``forward`` keeps what ``backward`` needs; decoding carries each layer's state and the
last inputs of its convolution, of one size however long the text has become.

    python examples/state_space_lm.py [--steps N] [--dtype bf16|f32]

trains on synthetic texts (each repeats a random phrase of its own) and prints the loss, then reads a prompt in
one pass and continues it by beam search.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_1810_09958_amd as isam  # noqa: E402
from recurrent_lm import loss_and_gradient, texts  # noqa: E402

_MATRICES = ("E", "Wi", "Wx", "Wdt", "Wo", "W1", "W2")     # in the model's dtype; the rest stays fp32


def init(vocab, D, inner, N, rank, F, layers, taps=4, device="cuda", seed=0):
    """Parameters in fp32: name -> tensor, layer l's as "l.name"."""
    g = torch.Generator().manual_seed(seed)

    def normal(rows, cols):
        return torch.randn((rows, cols), generator=g) * cols ** -0.5

    p = {"E": normal(vocab, D), "w_out": torch.ones(D)}
    for l in range(layers):
        step = torch.exp(torch.linspace(math.log(1e-3), math.log(1e-1), inner))
        layer = {"w0": torch.ones(D), "w1": torch.ones(D), "Wi": normal(2 * inner, D), "wc": normal(taps, inner), "bc": torch.zeros(inner),
                 "Wx": normal(rank + 2 * N, inner), "Wdt": normal(inner, rank), "dt_bias": torch.log(torch.expm1(step)),
                 "A_log": torch.log(torch.arange(1.0, N + 1)).expand(inner, N).contiguous(), "skip": torch.ones(inner), "Wo": normal(D, inner),
                 "W1": normal(F, D), "b1": torch.zeros(F), "W2": normal(D, F), "b2": torch.zeros(D)}
        p.update({f"{l}.{k}": v for k, v in layer.items()})
    return {k: v.to(device) for k, v in p.items()}


def cast(params, dtype):
    """The copies that the operators read."""
    return {k: v.to(dtype) if k.split(".")[-1] in _MATRICES else v for k, v in params.items()}


def layer_count(p):
    return 1 + max(int(k.split(".")[0]) for k in p if "." in k)


def sizes(p):
    """inner, N, rank and taps of the model."""
    return p["0.Wdt"].shape[0], p["0.A_log"].shape[1], p["0.Wdt"].shape[1], p["0.wc"].shape[0]


def empty_state(p, B):
    inner, N, _, taps = sizes(p)
    L, dev = layer_count(p), p["E"].device
    return torch.zeros((L, taps - 1, B, inner), device=dev, dtype=p["E"].dtype), torch.zeros((L, B, inner, N), device=dev)


def forward(p, tokens, state=None, reset=None, train=False):
    """tokens [T][batch]; state as this call returns it, or None; reset [T][batch] bool: a new text starts.
    Returns (logits [T * batch][vocab] fp32, the state after the last token, what ``backward`` needs)."""
    T, B = tokens.shape
    inner, N, rank, _ = sizes(p)
    state = state if state is not None else empty_state(p, B)
    after = tuple(torch.empty_like(s) for s in state)
    r = p["E"][tokens.reshape(-1)]
    saved = []
    for l in range(layer_count(p)):
        q = {k: p[f"{l}.{k}"] for k in ("w0", "w1", "Wi", "wc", "bc", "Wx", "Wdt", "dt_bias", "A_log", "skip", "Wo", "W1", "b1", "W2", "b2")}
        _, y0 = isam.norm_residual(None, r, w_pre=q["w0"])
        xz = isam.linear(y0, q["Wi"]).view(T, B, 2 * inner)
        x, _ = isam.causal_conv(xz[..., :inner], q["wc"], bias=q["bc"], state=state[0][l], reset=reset, state_T=after[0][l])
        sbc = isam.linear(x.view(T * B, inner), q["Wx"])
        dt = isam.linear(sbc[:, :rank], q["Wdt"]).view(T, B, inner)
        bc = sbc[:, rank:].view(T, B, 2 * N)
        A = -torch.exp(q["A_log"])
        kept = torch.empty(isam.selective_scan_states_shape(T, B, inner, N), device=r.device) if train else None
        h, _ = isam.selective_scan(x, dt, A, bc[..., :N], bc[..., N:], skip=q["skip"], z=xz[..., inner:], dt_bias=q["dt_bias"],
                                   h0=state[1][l], reset=reset, h_T=after[1][l], states=kept)
        r1 = isam.linear(h.view(T * B, inner), q["Wo"], residual=r)
        _, y1 = isam.norm_residual(None, r1, w_pre=q["w1"])
        u = isam.linear(y1, q["W1"], bias=q["b1"], activation="gelu")
        r2 = isam.linear(u, q["W2"], bias=q["b2"], residual=r1)
        if train:
            saved.append((q, state[0][l], r, y0, xz, x, sbc, dt, A, kept, h, r1, y1, u))
        r = r2
    _, y = isam.norm_residual(None, r, w_pre=p["w_out"])
    logits = isam.gemm(y, p["E"], trans_b=True)
    return logits, after, (tokens, reset, r, y, saved) if train else None


def backward(p, kept, dlogits):
    """Gradients of every parameter (fp32) from dlogits [T * batch][vocab]."""
    tokens, reset, r, y, saved = kept
    T, B = tokens.shape
    inner, N, rank, _ = sizes(p)
    dt_ = p["E"].dtype
    dlogits = dlogits.to(dt_)
    grad = {"E": isam.gemm(dlogits, y, trans_a=True)}
    dy = isam.gemm(dlogits, p["E"], out_dtype=dt_)
    _, dr, _, _, grad["w_out"] = isam.norm_residual_backward(None, r, dy, w_pre=p["w_out"])
    for l in reversed(range(layer_count(p))):
        q, state, r, y0, xz, x, sbc, dt, A, states, h, r1, y1, u = saved[l]
        g = {}
        du, g["W2"], g["b2"] = isam.linear_backward(u, q["W2"], dr, bias=q["b2"])
        dy, g["W1"], g["b1"] = isam.linear_backward(y1, q["W1"], du, bias=q["b1"], activation="gelu")
        _, dr, _, _, g["w1"] = isam.norm_residual_backward(None, r1, dy, dr_out=dr, w_pre=q["w1"])
        dh, g["Wo"], _ = isam.linear_backward(h.view(T * B, inner), q["Wo"], dr)
        dxz, dsbc = torch.empty_like(xz), torch.empty_like(sbc)
        bc, dbc = sbc[:, rank:].view(T, B, 2 * N), dsbc[:, rank:].view(T, B, 2 * N)
        dx, ddt, dA, _, _, g["skip"], _, g["dt_bias"], _ = isam.selective_scan_backward(
            x, dt, A, bc[..., :N], bc[..., N:], dh.view(T, B, inner), states=states, skip=q["skip"], z=xz[..., inner:],
            dt_bias=q["dt_bias"], reset=reset, dB=dbc[..., :N], dC=dbc[..., N:], dz=dxz[..., inner:])
        g["A_log"] = dA * A
        _, g["Wdt"], _ = isam.linear_backward(sbc[:, :rank], q["Wdt"], ddt.view(T * B, inner), dx=dsbc[:, :rank])
        dx2, g["Wx"], _ = isam.linear_backward(x.view(T * B, inner), q["Wx"], dsbc)
        _, _, g["wc"], g["bc"] = isam.causal_conv_backward(xz[..., :inner], q["wc"], dx + dx2.view(T, B, inner), bias=q["bc"], state=state,
                                                           reset=reset, dx=dxz[..., :inner])
        dy, g["Wi"], _ = isam.linear_backward(y0, q["Wi"], dxz.view(T * B, 2 * inner))
        _, dr, _, _, g["w0"] = isam.norm_residual_backward(None, r, dy, dr_out=dr, w_pre=q["w0"])
        grad.update({f"{l}.{k}": v.float() for k, v in g.items()})
    grad["E"].index_add_(0, tokens.reshape(-1), dr.float())
    return grad


def beam_decode(p, tokens, count, beams, end=-1):
    """Reads a prompt [T][batch] in one pass, then continues it by `count` tokens with the best `beams` texts of each.
    Returns (tokens [batch][beams][count], the best first, their log probabilities [batch][beams])."""
    B = tokens.shape[1]
    logits, state, _ = forward(p, tokens)
    logits = logits[-B:].view(B, 1, -1)
    scores, finished = torch.zeros((B, 1), device=tokens.device), None
    out = None
    for _ in range(count):
        scores, parent, token, finished = isam.beam_step(logits, scores, width=beams, finished=finished if end >= 0 else None, end=end)
        state = isam.beam_reorder(state[0], parent, dim=2), isam.beam_reorder(state[1], parent, dim=1)
        new = token.view(B * beams, 1)
        out = new if out is None else torch.cat((isam.beam_reorder(out, parent), new), 1)
        logits, state, _ = forward(p, token.view(1, B * beams), state)
        logits = logits.view(B, beams, -1)
    return out.view(B, beams, count), scores


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=400)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args()
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[a.dtype]
    vocab, T, B, phrase = 256, 512, 16, 8
    params = init(vocab, D=256, inner=512, N=16, rank=16, F=512, layers=2)
    opt = torch.optim.Adam(list(params.values()), lr=3e-3)
    g = torch.Generator().manual_seed(1)
    begin = 0.0
    for i in range(a.steps):
        if i == 5:
            torch.cuda.synchronize()
            begin = time.perf_counter()
        tokens, reset = texts(T, B, vocab, phrase, g, "cuda")
        p = cast(params, dtype)
        logits, _, kept = forward(p, tokens[:-1], reset=reset[:-1], train=True)
        loss, dlogits = loss_and_gradient(logits, tokens[1:].reshape(-1))
        grad = backward(p, kept, dlogits)
        for k, v in params.items():
            v.grad = grad[k]
        opt.step()
        if i % 50 == 0 or i == a.steps - 1:
            print(f"step {i}: loss {float(loss):.4f}", flush=True)
    torch.cuda.synchronize()
    if a.steps > 5:
        print(f"{(a.steps - 5) * T * B / (time.perf_counter() - begin):.0f} tokens/s in training")
    p = cast(params, dtype)
    words = torch.randint(vocab, (phrase, B), generator=g).cuda()
    out, scores = beam_decode(p, words.repeat(2, 1), 2 * phrase, beams=4)
    print(f"{float((out[:, 0].t() == words.repeat(2, 1)).float().mean()):.3f} of the best beams' tokens continue the phrase")


if __name__ == "__main__":
    main()
