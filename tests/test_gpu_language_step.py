"""The operators of a language model's step used together: lookup, layer norm, log probabilities, their gradients into workers' flat
vectors, the exchange, AdamW for what is no matrix and the orthogonalised update for what is.

The gradient is compared with 64 bits by the chain rule written out on the host.  Its tolerance: every stage is a handful of
float32 roundings of its own size, the products sum up to 48 terms, so 200 u of the gradient's largest element covers them all,
u = 2^-24, as in the test of the smaller example.
"""

import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_language", os.path.join(ROOT, "examples", "train_language.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradient_against_64_bits_and_differences(example):
    import torch

    net = example.Network(vocab=23, width=16, hidden=48)
    gen = torch.Generator(device="cuda").manual_seed(4)
    w = torch.randn(net.n, generator=gen, device="cuda") * 0.5
    net.view(w, net.gamma).add_(1.0)
    tokens = torch.randint(0, 23, (40,), generator=gen, device="cuda")
    targets = torch.randint(-1, 23, (40,), generator=gen, device="cuda")
    grad = torch.full((net.n,), 9.0, device="cuda")
    ops = example.Operators(net, 40)
    example.worker_gradient(net, ops, w, grad, tokens, targets, True)

    def loss(v):  # in 64 bits, on the host
        f = lambda p: net.view(v, p)  # noqa: E731
        x = f(net.table)[tokens.cpu()] * net.scale
        d = x - x.mean(1, keepdim=True)
        y = d / (d.square().mean(1, keepdim=True) + 1e-5).sqrt() * f(net.gamma) + f(net.beta)
        logits = torch.relu(y @ f(net.w1).t()) @ f(net.w2).t()
        logp = torch.log_softmax(logits, 1)
        t = targets.cpu()
        own = logp.gather(1, t.clamp(min=0).view(-1, 1)).view(-1)[t >= 0].sum()
        entropy = -(logp.exp() * logp).sum()
        return -(own + net.entropy_weight * entropy) / 40

    v = w.cpu().double().requires_grad_()
    loss(v).backward()
    scale = float(v.grad.abs().max())
    assert float((grad.cpu().double() - v.grad).abs().max()) <= 200 * 2.0 ** -24 * scale
    for i in torch.randperm(net.n, generator=torch.Generator().manual_seed(1))[:12].tolist():
        up, down = w.cpu().double(), w.cpu().double()
        up[i] += 1e-6
        down[i] -= 1e-6
        assert abs(float(loss(up) - loss(down)) / 2e-6 - float(grad[i])) <= 200 * 2.0 ** -24 * scale + 1e-7
    twice = grad.clone()
    example.worker_gradient(net, ops, w, twice, tokens, targets, False)
    assert torch.allclose(twice, 2 * grad, rtol=1e-6, atol=1e-7 * scale)
    ops.tokens.status()


def test_runs_and_the_same_twice(example):
    for bits in (32, 8):
        one, two = (example.train(steps=5, seed=3, state_bits=bits) for _ in range(2))
        assert one == two and all(math.isfinite(v) for v in one)


def test_answers(example):
    """A trained network's answer: single tokens with alternatives, as many as asked for, most likely first."""
    import torch

    net = example.Network(vocab=23, width=16, hidden=48)
    w = torch.randn(net.n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * 0.3
    chosen, alternatives = example.answer(net, w, first=5, length=6, top=4)
    assert len(chosen) == 6 and all(0 <= c < 23 for c in chosen)
    for token, (ids, logps) in zip(chosen, alternatives):
        assert ids[0] == token and sorted(logps, reverse=True) == logps and len(set(ids)) == 4
        assert all(v <= 0.0 for v in logps)
