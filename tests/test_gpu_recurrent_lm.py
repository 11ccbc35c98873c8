"""The example model (all operators together) against the same model in 64 bits.

Bounds: every fp32 product here has at most K = 80 terms and every sum over rows at most 150, so an operator
adds at most some 150 u (u = 2^-24) relative to the norm of its result; a path through the model and back
passes 2 layers x 4 products and norms, twice, 16 operators, and a norm's or an activation's factors can
raise an error by a few: 4 x 16 x 150 u = 2^-10.7 of the norm of each output."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
BOUND = 4 * 16 * 150 * 2.0 ** -24


@pytest.fixture(scope="module")
def lm():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "recurrent_lm.py")
    spec = importlib.util.spec_from_file_location("recurrent_lm", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def setup(lm, T, B, dtype):
    p = lm.init(50, 40, 72, 80, 2, seed=T)
    g = torch.Generator().manual_seed(T)
    for k, v in p.items():      # nothing left at one or zero
        v += (torch.randn(v.shape, generator=g) * 0.1).cuda()
    tokens = torch.randint(50, (T + 1, B), generator=g).cuda()
    return lm.cast(p, dtype), tokens, (torch.rand((T, B), generator=g) < 0.05).cuda()


def reference(p, tokens, targets, reset):
    """Logits, loss and gradients by automatic differentiation in 64 bits on the CPU."""
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in p.items()}
    tokens, targets = tokens.cpu(), targets.cpu()
    T, B = tokens.shape

    def rms(v):
        return v / (v.pow(2).mean(1, keepdim=True) + 1e-6).sqrt()

    r = p["E"][tokens.reshape(-1)]
    y = rms(r) * p["w_in"]
    for l in range(2):
        q = {k[2:]: v for k, v in p.items() if k.startswith(f"{l}.")}
        H = q["Wo"].shape[1]
        gx = (y @ q["Wi"].t() + q["bi"]).view(T, B, 2 * H)
        h, hs = torch.zeros((B, H), dtype=torch.float64), []
        for t in range(T):
            if reset is not None:
                h = torch.where(reset[t].cpu()[:, None], 0.0, h)
            z = torch.sigmoid(gx[t, :, :H])
            h = z * h + (1 - z) * torch.tanh(gx[t, :, H:])
            hs.append(h)
        x = torch.cat(hs) @ q["Wo"].t()
        r = r + q["gate0"] * rms(x) * q["w_post0"]
        y = rms(r) * q["w_pre0"]
        gu = y @ q["W"].t() + q["b"]
        F = gu.shape[1] // 2
        x = (torch.nn.functional.silu(gu[:, :F]) * gu[:, F:]) @ q["Wd"].t()
        r = r + q["gate1"] * rms(x) * q["w_post1"]
        y = rms(r) * q["w_pre1"]
    logits = y @ p["E"].t()
    loss = torch.nn.functional.cross_entropy(logits, targets.reshape(-1))
    loss.backward()
    return logits.detach(), loss.detach(), {k: v.grad for k, v in p.items()}


def close(got, ref, name, bound):
    err = float((got.cpu().double() - ref).norm() / ref.norm())
    assert err <= bound, f"{name}: {err:.2e} above {bound:.2e}"


@pytest.mark.parametrize("T,B", [(1, 1), (9, 3), (150, 1)])
def test_training_step(lm, T, B):
    p, tokens, reset = setup(lm, T, B, torch.float32)
    want = reference(p, tokens[:-1], tokens[1:], reset)
    logits, _, kept = lm.forward(p, tokens[:-1], reset=reset, train=True)
    loss, dlogits = lm.loss_and_gradient(logits, tokens[1:].reshape(-1))
    close(logits, want[0], "logits", BOUND)
    close(loss, want[1], "loss", BOUND)
    grad = lm.backward(p, kept, dlogits)
    assert grad.keys() == want[2].keys()
    for k, v in grad.items():
        close(v, want[2][k], k, BOUND)


def test_decoding_token_by_token(lm):
    # the logits of each decoded token are those of one pass over the whole text
    p, tokens, _ = setup(lm, 70, 3, torch.float32)
    out, seen = lm.decode(p, tokens[:-1], 12)
    whole, _, _ = lm.forward(p, torch.cat((tokens[:-1], out)))
    whole = whole.view(82, 3, -1)[69:81]
    close(seen, whole.cpu().double(), "logits", 2 * BOUND)


def test_bf16_training_lowers_the_loss(lm):
    params = lm.init(50, 64, 64, 128, 1, seed=3)
    opt = torch.optim.Adam(list(params.values()), lr=3e-3)
    g = torch.Generator().manual_seed(2)
    tokens, reset = lm.texts(64, 8, 50, 4, g, "cuda")
    losses = []
    for _ in range(30):
        p = lm.cast(params, torch.bfloat16)
        logits, _, kept = lm.forward(p, tokens[:-1], reset=reset[:-1], train=True)
        loss, dlogits = lm.loss_and_gradient(logits, tokens[1:].reshape(-1))
        losses.append(float(loss))
        for k, v in lm.backward(p, kept, dlogits).items():
            params[k].grad = v
        opt.step()
    assert losses[-1] < 0.5 * losses[0], losses
