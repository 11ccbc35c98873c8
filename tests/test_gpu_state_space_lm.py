"""The example models with the state-space block's operators and beam search together, against the same models in 64 bits.

Bounds: every fp32 product here has at most K = 96 terms and every sum over rows at most 150, so an operator adds at
most some 150 u (u = 2^-24) relative to the norm of its result (the scan, whose states live for some tens of tokens
here, a few such); a path through the model and back passes 2 layers x 9 operators, twice, 36, and their factors can
raise an error by a few: 4 x 36 x 150 u = 2^-9.6 of the norm of each output."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
BOUND = 4 * 36 * 150 * 2.0 ** -24


def load(name):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", name + ".py")
    spec = importlib.util.spec_from_file_location(name, path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.fixture(scope="module")
def lm():
    return load("state_space_lm")


def setup(lm, T, B, dtype):
    p = lm.init(50, 40, 48, 8, 6, 96, 2, seed=T)
    g = torch.Generator().manual_seed(T)
    for k, v in p.items():      # nothing left at one or zero
        v += (torch.randn(v.shape, generator=g) * 0.1).cuda()
    tokens = torch.randint(50, (T + 1, B), generator=g).cuda()
    return lm.cast(p, dtype), tokens, (torch.rand((T, B), generator=g) < 0.05).cuda()


def logits_of(p, tokens, reset):
    """Logits [T][batch][vocab] in 64 bits on the CPU, token by token."""
    T, B = tokens.shape

    def rms(v):
        return v / (v.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()

    r = p["E"][tokens]
    for l in range(2):
        q = {k[2:]: v for k, v in p.items() if k.startswith(f"{l}.")}
        inner, N = q["A_log"].shape
        rank, K = q["Wdt"].shape[1], q["wc"].shape[0]
        xz = (rms(r) * q["w0"]) @ q["Wi"].t()
        window = [torch.zeros((B, inner), dtype=torch.float64)] * (K - 1)
        h = torch.zeros((B, inner, N), dtype=torch.float64)
        ys = []
        for t in range(T):
            keep = torch.ones((B, 1), dtype=torch.float64) if reset is None else (~reset[t]).double()[:, None]
            window = [v * keep for v in window[-(K - 1):]] + [xz[t, :, :inner]]
            x = torch.nn.functional.silu(q["bc"] + sum(q["wc"][k] * window[k] for k in range(K)))
            sbc = x @ q["Wx"].t()
            d = torch.nn.functional.softplus(sbc[:, :rank] @ q["Wdt"].t() + q["dt_bias"], threshold=100)
            h = torch.exp(d[..., None] * -torch.exp(q["A_log"])) * (h * keep[..., None]) + (d * x)[..., None] * sbc[:, None, rank:rank + N]
            ys.append(((h * sbc[:, None, rank + N:]).sum(-1) + q["skip"] * x) * torch.nn.functional.silu(xz[t, :, inner:]))
        r = r + torch.stack(ys) @ q["Wo"].t()
        u = (rms(r) * q["w1"]) @ q["W1"].t() + q["b1"]
        r = r + (u * 0.5 * torch.erfc(-u / math.sqrt(2))) @ q["W2"].t() + q["b2"]
    return (rms(r) * p["w_out"]) @ p["E"].t()


def close(got, ref, name, bound):
    err, norm = float((got.cpu().double() - ref).norm()), float(ref.norm())   # (a gradient may be all zeros)
    assert err <= bound * norm, f"{name}: {err:.2e} of {norm:.2e}, above {bound:.2e}"


@pytest.mark.parametrize("T,B", [(1, 1), (9, 3), (150, 1), (40, 2)])
def test_training_step(lm, T, B):
    p, tokens, reset = setup(lm, T, B, torch.float32)
    ref = {k: v.detach().cpu().double().requires_grad_() for k, v in p.items()}
    want = logits_of(ref, tokens[:-1].cpu(), reset.cpu()).reshape(T * B, -1)
    want_loss = torch.nn.functional.cross_entropy(want, tokens[1:].cpu().reshape(-1))
    want_loss.backward()
    logits, _, kept = lm.forward(p, tokens[:-1], reset=reset, train=True)
    loss, dlogits = lm.loss_and_gradient(logits, tokens[1:].reshape(-1))
    close(logits, want.detach(), "logits", BOUND)
    close(loss, want_loss.detach(), "loss", BOUND)
    grad = lm.backward(p, kept, dlogits)
    assert grad.keys() == ref.keys()
    for k, v in grad.items():
        close(v, ref[k].grad, k, BOUND)


def test_tokens_one_by_one(lm):
    # a prompt in one pass, then token by token: the logits of one pass over all
    p, tokens, _ = setup(lm, 60, 3, torch.float32)
    whole = lm.forward(p, tokens)[0].view(61, 3, -1)
    logits, state, _ = lm.forward(p, tokens[:40])
    seen = [logits.view(40, 3, -1)[-1]]
    for t in range(40, 61):
        logits, state, _ = lm.forward(p, tokens[t:t + 1], state)
        seen.append(logits)
    close(torch.stack(seen), whole[39:].cpu().double(), "logits", 2 * BOUND)


def search(logits_of_text, prompt, count, beams, end):
    """Beam search over one prompt in 64 bits, its texts evaluated whole."""
    alive = [(0.0, [], False)]
    for _ in range(count):
        found = []
        for i, (score, text, done) in enumerate(alive):
            if done:
                found.append((score, text + [end], True))
                continue
            logp = torch.log_softmax(logits_of_text(prompt + text), 0)
            found += [(score + float(v), text + [j], j == end) for j, v in enumerate(logp)]
        alive = sorted(found, key=lambda f: -f[0])[:beams]
    return alive


@pytest.mark.parametrize("end", [-1, 3])
def test_beam_search(lm, end):
    p, tokens, _ = setup(lm, 12, 2, torch.float32)
    ref = {k: v.detach().cpu().double() for k, v in p.items()}
    out, scores = lm.beam_decode(p, tokens, 4, beams=3, end=end)
    for b in range(2):
        best = search(lambda text: logits_of(ref, torch.tensor(text)[:, None], None)[-1, 0], tokens[:, b].tolist(), 4, 3, end)
        assert out[b].tolist() == [t for _, t, _ in best]
        close(scores[b], torch.tensor([s for s, _, _ in best], dtype=torch.float64), "scores", BOUND)


def test_beam_search_of_the_recurrent_model():
    m = load("recurrent_lm")
    p = m.cast(m.init(50, 40, 72, 80, 2, seed=3), torch.float32)
    tokens = torch.randint(50, (10, 2), generator=torch.Generator().manual_seed(1)).cuda()
    one, _ = m.beam_decode(p, tokens, 5, beams=1)
    assert torch.equal(one[:, 0].t().long(), m.decode(p, tokens, 5)[0])       # one beam: the likeliest token each time
    for end in (-1, 3):
        out, scores = m.beam_decode(p, tokens, 4, beams=3, end=end)
        for b in range(2):
            best = search(lambda text: m.forward(p, torch.tensor(text, device="cuda")[:, None])[0][-1].cpu().double(), tokens[:, b].tolist(),
                          4, 3, end)
            assert out[b].tolist() == [t for _, t, _ in best]
            close(scores[b], torch.tensor([s for s, _, _ in best], dtype=torch.float64), "scores", BOUND)


def test_bf16_runs_and_a_state_of_one_size(lm):
    p, tokens, reset = setup(lm, 64, 4, torch.bfloat16)
    logits, state, kept = lm.forward(p, tokens[:-1], reset=reset, train=True)
    grad = lm.backward(p, kept, torch.randn_like(logits) / len(logits))
    assert all(torch.isfinite(v).all() and v.shape == p[k].shape for k, v in grad.items())
    one = lm.forward(p, tokens[:1])[1]
    assert [s.shape for s in state] == [s.shape for s in one]
