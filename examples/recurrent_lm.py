"""A small language model of gated recurrent blocks, trained and decoded with the library's operators.

    r_0 = E[token],                     y_0 = norm(r_0)
    x   = linear_gru(y Wi^T) Wo^T       then  r, y = norm_residual(x, r)      (each layer's first half)
    x   = gated_ffn(y) Wd^T             then  r, y = norm_residual(x, r)      (its second half)
    logits = y E^T

Activations are rows [T * batch][D], time first, so one call covers a prompt, a training step or (T = 1)
one token of every sequence.  ``forward`` keeps what ``backward`` needs; ``decode`` carries only each
layer's state, [batch][H] in fp32, however long the text has become.

    python examples/recurrent_lm.py [--steps N] [--dtype bf16|f32]

trains on synthetic texts (each repeats a random phrase of its own) and prints the loss, then reads a
prompt in one pass and continues it token by token.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1810_09958_amd as isam  # noqa: E402

_MATRICES = ("E", "Wi", "Wo", "W", "Wd", "gate")     # in the model's dtype; the rest stays fp32


def init(vocab, D, H, F, layers, device="cuda", seed=0):
    """Parameters in fp32: name -> tensor, layer l's as "l.name"."""
    g = torch.Generator().manual_seed(seed)

    def normal(rows, cols):
        return torch.randn((rows, cols), generator=g) * cols ** -0.5

    p = {"E": normal(vocab, D), "w_in": torch.ones(D)}
    for l in range(layers):
        layer = {"Wi": normal(2 * H, D), "bi": torch.cat((torch.linspace(0, 5, H), torch.zeros(H))), "Wo": normal(D, H),
                 "W": normal(2 * F, D), "b": torch.zeros(2 * F), "Wd": normal(D, F)}
        for half in "01":
            layer.update({"gate" + half: torch.full((1, D), 0.5), "w_post" + half: torch.ones(D), "w_pre" + half: torch.ones(D)})
        p.update({f"{l}.{k}": v for k, v in layer.items()})
    return {k: v.to(device) for k, v in p.items()}


def cast(params, dtype):
    """The copies that the operators read."""
    return {k: v.to(dtype) if k.split(".")[-1].rstrip("01") in _MATRICES else v for k, v in params.items()}


def layer_count(p):
    return 1 + max(int(k.split(".")[0]) for k in p if "." in k)


def _norm_args(p, l, half):
    return dict(w_post=p[f"{l}.w_post{half}"], w_pre=p[f"{l}.w_pre{half}"], gate=p[f"{l}.gate{half}"])


def forward(p, tokens, state=None, reset=None, train=False):
    """tokens [T][batch]; state [layers][batch][H] fp32 or None; reset [T][batch] bool: a new text starts.
    Returns (logits [T * batch][vocab] fp32, the state after the last token, what ``backward`` needs)."""
    T, B = tokens.shape
    H = p["0.Wo"].shape[1]
    layers, dt = layer_count(p), p["E"].dtype
    out_state = torch.empty((layers, B, H), device=tokens.device)
    r, y = isam.norm_residual(None, p["E"][tokens.reshape(-1)], w_pre=p["w_in"])
    saved = [(r,)]
    for l in range(layers):
        gx = isam.gemm(y, p[f"{l}.Wi"], trans_b=True, out_dtype=dt).view(T, B, 2 * H)
        states = torch.empty(isam.linear_gru_states_shape(T, B, H), device=tokens.device) if train else None
        h, _ = isam.linear_gru(gx, bias=p[f"{l}.bi"], h0=None if state is None else state[l], reset=reset, h_T=out_state[l],
                               states=states)
        h = h.view(T * B, H)
        x = isam.gemm(h, p[f"{l}.Wo"], trans_b=True, out_dtype=dt)
        y0 = y
        r, y = isam.norm_residual(x, r, **_norm_args(p, l, 0))
        u = isam.gated_ffn(y, p[f"{l}.W"], bias=p[f"{l}.b"])
        x1 = isam.gemm(u, p[f"{l}.Wd"], trans_b=True, out_dtype=dt)
        r1, y1 = isam.norm_residual(x1, r, **_norm_args(p, l, 1))
        if train:
            saved.append((y0, gx, states, h, x, r, y, u, x1, r1))
        r, y = r1, y1
    logits = isam.gemm(y, p["E"], trans_b=True)
    return logits, out_state, (tokens, reset, y, saved) if train else None


def backward(p, kept, dlogits):
    """Gradients of every parameter (fp32) from dlogits [T * batch][vocab]."""
    tokens, reset, y, saved = kept
    T, B = tokens.shape
    dt = p["E"].dtype
    dlogits = dlogits.to(dt)
    grad = {"E": isam.gemm(dlogits, y, trans_a=True)}
    dy, dr = isam.gemm(dlogits, p["E"], out_dtype=dt), None
    for l in reversed(range(layer_count(p))):
        y0, gx, states, h, x, r, y, u, x1, r1 = saved[l + 1]
        H = h.shape[1]

        def norm(x, r, dy, dr, half):
            dx, dr, *rest = isam.norm_residual_backward(x, r, dy, dr_out=dr, **_norm_args(p, l, half))
            for k, v in zip(("gate", "w_post", "w_pre"), rest):
                grad[f"{l}.{k}{half}"] = v.float()
            return dx, dr

        dx, dr = norm(x1, r1, dy, dr, 1)
        grad[f"{l}.Wd"] = isam.gemm(dx, u, trans_a=True)
        du = isam.gemm(dx, p[f"{l}.Wd"], out_dtype=dt)
        dy, dW, grad[f"{l}.b"] = isam.gated_ffn_backward(y, p[f"{l}.W"], du, bias=p[f"{l}.b"])
        grad[f"{l}.W"] = dW.float()
        dx, dr = norm(x, r, dy, dr, 0)
        grad[f"{l}.Wo"] = isam.gemm(dx, h, trans_a=True)
        dh = isam.gemm(dx, p[f"{l}.Wo"], out_dtype=dt).view(T, B, H)
        dgx, _, grad[f"{l}.bi"] = isam.linear_gru_backward(gx, dh, states=states, bias=p[f"{l}.bi"], reset=reset)
        dgx = dgx.view(T * B, 2 * H)
        grad[f"{l}.Wi"] = isam.gemm(dgx, y0, trans_a=True)
        dy = isam.gemm(dgx, p[f"{l}.Wi"], out_dtype=dt)
    _, dr, _, _, grad["w_in"] = isam.norm_residual_backward(None, saved[0][0], dy, dr_out=dr, w_pre=p["w_in"])
    grad["E"].index_add_(0, tokens.reshape(-1), dr.float())
    return grad


def loss_and_gradient(logits, targets):
    """Mean cross entropy of targets [T * batch] and its gradient with respect to the logits."""
    logp = torch.log_softmax(logits, 1)
    d = logp.exp()
    d[torch.arange(len(targets), device=targets.device), targets] -= 1
    return -logp.gather(1, targets[:, None]).mean(), d / len(targets)


def decode(p, tokens, count):
    """Reads a prompt [T][batch] in one pass, then `count` tokens one by one (the likeliest each time).
    Returns the tokens [count][batch] and their logits [count][batch][vocab]."""
    B = tokens.shape[1]
    logits, state, _ = forward(p, tokens)
    out, seen = [], []
    for _ in range(count):
        seen.append(logits[-B:])
        out.append(seen[-1].argmax(1))
        logits, state, _ = forward(p, out[-1][None], state)
    return torch.stack(out), torch.stack(seen)


def texts(T, B, vocab, phrase, generator, device):
    """Packed texts [T + 1][batch], each repeating a random phrase of its own; reset marks where one starts."""
    t = torch.arange(T + 1)
    which, at = t // (4 * phrase), t % phrase
    words = torch.randint(vocab, (B, int(which[-1]) + 1, phrase), generator=generator)
    return words[:, which, at].t().contiguous().to(device), (t % (4 * phrase) == 0)[:, None].expand(T + 1, B).contiguous().to(device)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=400)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args()
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[a.dtype]
    vocab, D, T, B, phrase = 256, 256, 512, 16, 8
    params = init(vocab, D, H=512, F=1024, layers=2)
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
    out, _ = decode(p, words.repeat(2, 1), 2 * phrase)
    print(f"{float((out == words.repeat(2, 1)).float().mean()):.3f} of the decoded tokens continue the phrase")


if __name__ == "__main__":
    main()
