"""Data-parallel training of a small network on one GPU, W workers simulated, every step by the library:

    each worker   forward and backward over its micro-batches; the layer norm's weight gradients land in the worker's flat
                  gradient vector (artopk_layernorm_forward, artopk_layernorm_backward)
    exchange      AR-Topk step on the flat gradients with error feedback, layer by layer (artopk_step)
    update        momentum, orthogonalised per weight matrix, decoupled decay; loose weights (gains, biases) by plain
                  momentum (artopk_muon_step)

The network is linear -> layer norm -> relu -> linear -> softmax; its linear layers are torch products.  Inputs are
drawn from a fixed random teacher, so the loss has something to learn.  Run:  python examples/train_step.py
"""

import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2312_02493_amd as artopk  # noqa: E402


class Network:
    """Places of the weights in a flat vector; a matrix is (offset, rows, cols), a vector (offset, length)."""

    def __init__(self, inputs: int, hidden: int, classes: int):
        self.inputs, self.hidden, self.classes = inputs, hidden, classes
        at = 0
        self.w1 = (at, hidden, inputs)
        at += hidden * inputs
        self.gamma = (at, hidden)
        at += hidden
        self.beta = (at, hidden)
        at += hidden
        self.w2 = (at, classes, hidden)
        at += classes * hidden
        self.b2 = (at, classes)
        self.n = at + classes
        self.bounds = [0, self.gamma[0], self.beta[0], self.w2[0], self.b2[0], self.n]  # layers, for the selection

    def view(self, flat, place):
        at, *shape = place
        return flat[at:at + math.prod(shape)].view(*shape)

    def matrices(self):
        return [(at, r, c, math.sqrt(max(1.0, r / c))) for at, r, c in (self.w1, self.w2)]


def worker_gradient(net, norm, weights, grad, x, labels, first: bool):
    """Adds a micro-batch's gradient to `grad` (overwrites it with `first`); the mean loss as a tensor."""
    rows = x.shape[0]
    w1, w2 = net.view(weights, net.w1), net.view(weights, net.w2)
    h = x @ w1.t()
    y = torch.empty_like(h)
    mean, rstd = torch.empty(rows, device=x.device), torch.empty(rows, device=x.device)
    norm.artopk_layernorm_forward(h, net.view(weights, net.gamma), net.view(weights, net.beta), y, mean, rstd)
    a = torch.relu(y)
    logits = a @ w2.t() + net.view(weights, net.b2)
    logp = torch.log_softmax(logits, 1)
    loss = -logp.gather(1, labels.view(-1, 1)).mean()
    d = logp.exp()
    d[torch.arange(rows, device=x.device), labels] -= 1.0
    d /= rows
    dy = (d @ w2) * (y > 0)
    dh = torch.empty_like(h)
    norm.artopk_layernorm_backward(dy, h, net.view(weights, net.gamma), mean, rstd, dh, net.view(grad, net.gamma),
                                   net.view(grad, net.beta), accumulate=not first)
    for place, g in ((net.w1, dh.t() @ x), (net.w2, d.t() @ a), (net.b2, d.sum(0))):
        view = net.view(grad, place)
        view.copy_(g) if first else view.add_(g)
    return loss


def train(steps: int = 60, workers: int = 4, batch: int = 128, micro: int = 2, inputs: int = 48, hidden: int = 160,
          classes: int = 10, keep: float = 0.1, eta: float = 0.05, seed: int = 0):
    """Losses of the steps, mean over the workers."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    net = Network(inputs, hidden, classes)
    teacher = torch.randn(classes, inputs, generator=gen, device=dev)
    weights = torch.zeros(net.n, device=dev)
    net.view(weights, net.w1).normal_(0.0, 1.0 / math.sqrt(inputs), generator=gen)
    net.view(weights, net.w2).normal_(0.0, 1.0 / math.sqrt(hidden), generator=gen)
    net.view(weights, net.gamma).fill_(1.0)
    grads = [torch.zeros(net.n, device=dev) for _ in range(workers)]
    residuals = [torch.zeros(net.n, device=dev) for _ in range(workers)]
    update, momentum = torch.zeros(net.n, device=dev), torch.zeros(net.n, device=dev)
    seg_k = [math.ceil(keep * (b - a)) for a, b in zip(net.bounds, net.bounds[1:])]
    k = sum(seg_k)
    idx, summed = torch.zeros(k, dtype=torch.int32, device=dev), torch.zeros(k, device=dev)
    norm = artopk.NormContext(batch, hidden)
    exchange = artopk.Context(workers, net.n, k, len(seg_k))
    muon = artopk.MatrixContext(net.matrices(), net.n)
    losses = []
    for step in range(1, steps + 1):
        total = torch.zeros((), device=dev)
        for g in grads:
            for m in range(micro):
                x = torch.randn(batch, inputs, generator=gen, device=dev)
                total += worker_gradient(net, norm, weights, g, x, (x @ teacher.t()).argmax(1), m == 0)
        exchange.artopk_step(grads, residuals, k, artopk.ARTOPK_STAR, step, idx, summed, update, seg_off=net.bounds, seg_k=seg_k)
        muon.artopk_muon_step(weights, momentum, update, eta=eta, mu=0.9, decay=0.01, eta_rest=eta,
                              update_scale=1.0 / (workers * micro))
        losses.append(total / (workers * micro))
    exchange.status()
    return [float(v) for v in losses]


if __name__ == "__main__":
    history = train()
    for i in range(0, len(history), 10):
        print(f"step {i + 1:3d}  loss {history[i]:.4f}")
    print(f"step {len(history):3d}  loss {history[-1]:.4f}")
