"""The training example: layer norm, exchange and orthogonalised update together.  Its gradient is that of its loss, and the
loss falls to well below where it starts (ln 10 = 2.30 for ten classes it knows nothing about)."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_step", os.path.join(ROOT, "examples", "train_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradient_against_differences(example):
    import torch
    import paper_2312_02493_amd as lib

    net = example.Network(7, 20, 5)
    gen = torch.Generator(device="cuda").manual_seed(4)
    w = torch.randn(net.n, generator=gen, device="cuda") * 0.5
    x = torch.randn(16, 7, generator=gen, device="cuda")
    labels = torch.randint(0, 5, (16,), generator=gen, device="cuda")
    norm = lib.NormContext(16, 20)
    g = torch.full((net.n,), 9.0, device="cuda")
    example.worker_gradient(net, norm, w, g, x, labels, True)

    def loss(v):  # in 64 bits, on the host
        f = lambda p: net.view(v, p)  # noqa: E731
        h = x.cpu().double() @ f(net.w1).t()
        d = h - h.mean(1, keepdim=True)
        y = d / (d.square().mean(1, keepdim=True) + 1e-5).sqrt() * f(net.gamma) + f(net.beta)
        logp = torch.log_softmax(torch.relu(y) @ f(net.w2).t() + f(net.b2), 1)
        return -logp.gather(1, labels.cpu().view(-1, 1)).mean()

    v = w.cpu().double().requires_grad_()
    loss(v).backward()
    scale = float(v.grad.abs().max())
    # some hundred float32 roundings of values of the gradient's size
    assert float((g.cpu().double() - v.grad).abs().max()) <= 200 * 2.0 ** -24 * scale
    at = torch.randperm(net.n, generator=torch.Generator().manual_seed(1))[:12]
    for i in at.tolist():
        up, down = w.cpu().double(), w.cpu().double()
        up[i] += 1e-6
        down[i] -= 1e-6
        assert abs(float(loss(up) - loss(down)) / 2e-6 - float(g[i])) <= 200 * 2.0 ** -24 * scale + 1e-7
    twice = g.clone()
    example.worker_gradient(net, norm, w, twice, x, labels, False)
    assert torch.allclose(twice, 2 * g, rtol=1e-6, atol=1e-7 * scale)


def test_loss_falls(example):
    history = example.train(steps=60)
    assert all(v == v for v in history)
    assert 1.8 < history[0] < 3.5
    assert sum(history[-5:]) / 5 < 0.5 * history[0], history[::10]


def test_runs_the_same_twice(example):
    assert example.train(steps=8, seed=3) == example.train(steps=8, seed=3)
