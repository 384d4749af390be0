"""The operators together, as the language model of examples/ runs them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "recurrent_lm.py")


@pytest.fixture(scope="module")
def lm():
    spec = importlib.util.spec_from_file_location("recurrent_lm", _PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _tokens(T, batch, words, seed=3):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randint(0, words, (T, batch), generator=gen, device="cuda")


def _off(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


# What two orders of summation may make of a value: bf16 results differ by a step of 2^-7 now and then, which takes an e4m3 value
# over its border, by a step of at most 2^-3, for at most a sixteenth of them (2^-7 / 2^-3).  So a product is off by at most
# 2^-3 sqrt(2^-4) = 2^-5 in norm; five products in quadrature 0.07.
ORDER = 0.1


def test_prompt_at_once_and_token_by_token(lm):
    import torch
    model = lm.RecurrentLm(700, 200, 2)
    tokens = _tokens(37, 3, 700)
    at_once, state = model.forward(tokens, last_only=True)
    now = None
    for t in range(37):
        logits, now = model.forward(tokens[t:t + 1], state=now)
    assert _off(logits, at_once) < ORDER and _off(now, state) < ORDER
    # prompts of different length in one batch: the state of each is that of the prompt alone
    lengths = torch.tensor([37, 1, 20], dtype=torch.int32, device="cuda")
    ragged, states = model.forward(tokens, lengths, last_only=True)
    for b, n in enumerate(lengths.tolist()):
        alone, own = model.forward(tokens[:n, b:b + 1].contiguous(), last_only=True)
        assert _off(ragged[b:b + 1], alone) < ORDER and _off(states[:, b:b + 1], own) < ORDER


def test_recorded_steps_write_what_eager_ones_do(lm):
    import torch
    model = lm.RecurrentLm(1000, 300, 2)
    logits, state = model.forward(_tokens(12, 5, 1000), last_only=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    u = torch.rand((20, 5), generator=gen, device="cuda")
    out = []
    for recorded in (False, True):
        writer = lm.Writer(model, logits.argmax(1), state, temperature=0.9, top_k=60, top_p=0.95, min_p=0.01)
        if recorded:
            writer.record()
        out.append(writer.write(u))
        out.append(writer.state)
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
    assert len(set(out[0].flatten().tolist())) > 20 and int(out[0].min()) >= 0 and int(out[0].max()) < 1000


def _plain_loss(p, tokens, targets, blocks, H):
    """The model without a rounding, in fp64."""
    import torch
    T, batch = tokens.shape

    def norm(s, w):
        return s * (s.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w

    x = p["embedding"][tokens]
    for k in range(blocks):
        P = norm(x, p[f"norm{k}"]) @ p[f"in{k}"].T + p[f"bias{k}"]
        f, i, o, g = P[..., :H].sigmoid(), P[..., H:2 * H].sigmoid(), P[..., 2 * H:3 * H].sigmoid(), P[..., 3 * H:].tanh()
        c, hs = torch.zeros(batch, H, dtype=torch.float64), []
        for t in range(T):
            c = f[t] * c + i[t] * g[t]
            hs.append(o[t] * c.tanh())
        x = x + torch.stack(hs) @ p[f"out{k}"].T
    logits = norm(x, p["norm"]) @ p["vocabulary"].T
    return torch.nn.functional.cross_entropy(logits.reshape(T * batch, -1), targets.reshape(-1))


def test_gradient_is_near_that_of_the_model_without_roundings(lm):
    import torch
    T, batch, words, H, blocks = 40, 2, 300, 160, 2
    model = lm.RecurrentLm(words, H, blocks)
    tokens, targets = _tokens(T, batch, words), _tokens(T, batch, words, 4)
    loss, grad = model.gradient(tokens, targets)
    p = {k: v.double().cpu().requires_grad_() for k, v in model.params.items()}
    plain = _plain_loss(p, tokens.cpu(), targets.cpu(), blocks, H)
    plain.backward()
    # A value of a block is off by 2^-4 of itself at most, about 2^-5.3 in quadrature over the values; a product of two such by 2^-4.8.
    # The way forward and back passes at most ten of them: 2^-4.8 sqrt(10) = 0.11; twice that.
    assert abs(float(loss) - float(plain.detach())) < 0.22 * float(plain.detach())
    for k, v in p.items():
        assert _off(grad[k].cpu(), v.grad) < 0.22, (k, _off(grad[k].cpu(), v.grad))


def test_it_learns(lm):
    model = lm.RecurrentLm(200, 128, 2)
    losses = lm.train(model, _tokens(33, 4, 200), 40, 2e-3)
    assert losses[0] > 4 and losses[-1] < losses[0] / 2
