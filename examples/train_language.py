"""Data-parallel training of a small language model on one GPU, W workers simulated, every step by the library:

    each worker   lookup of its tokens' rows (artopk_embedding_forward), layer norm, two linear layers, log probabilities of the
                  next tokens with the entropy as a bonus (artopk_token_logprobs); then the gradients of all of these, which land
                  in the worker's flat gradient vector
    exchange      AR-Topk step on the flat gradients with error feedback, layer by layer (artopk_step)
    update        the linear layers by the orthogonalised momentum step (artopk_muon_step), the embedding and the gains by AdamW
                  (artopk_adamw_step), moments in 8 bits
    answers       token by token, with the most likely alternatives (artopk_token_logprobs)

The linear layers' products are torch's.  The text is drawn from a fixed random table of which token follows which, so there is
something to learn.  Run:  python examples/train_language.py
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
    """embedding -> layer norm -> linear -> relu -> linear; places of the weights in a flat vector."""

    def __init__(self, vocab: int, width: int, hidden: int, entropy_weight: float = 0.01):
        self.vocab, self.width, self.hidden, self.entropy_weight = vocab, width, hidden, entropy_weight
        self.scale = math.sqrt(width)
        at, self.bounds = 0, [0]
        for name, shape in (("table", (vocab, width)), ("gamma", (width,)), ("beta", (width,)), ("w1", (hidden, width)),
                            ("w2", (vocab, hidden))):
            setattr(self, name, (at, *shape))
            at += math.prod(shape)
            self.bounds.append(at)
        self.n = at

    def view(self, flat, place):
        at, *shape = place
        return flat[at:at + math.prod(shape)].view(*shape)

    def matrices(self):
        return [(at, r, c, math.sqrt(max(1.0, r / c))) for at, r, c in (self.w1, self.w2)]

    def tensors(self):
        """What AdamW moves: the embedding, decayed, and the layer norm's weights."""
        (table, rows, cols), (gamma, width), (beta, _) = self.table, self.gamma, self.beta
        return [(table, rows * cols, 1.0, 0.01), (gamma, width, 1.0, 0.0), (beta, width, 1.0, 0.0)]


class Operators:
    """The handles of a worker's pass over up to `rows` tokens."""

    def __init__(self, net: Network, rows: int):
        self.tokens = artopk.TokenContext(rows, net.vocab, net.width)
        self.norm = artopk.NormContext(rows, net.width)


def forward(net, ops, weights, tokens):
    """(embedded, normalised, mean, rstd, hidden, logits) of a batch of tokens."""
    rows, dev = tokens.shape[0], weights.device
    x, y = torch.empty(rows, net.width, device=dev), torch.empty(rows, net.width, device=dev)
    mean, rstd = torch.empty(rows, device=dev), torch.empty(rows, device=dev)
    ops.tokens.artopk_embedding_forward(net.view(weights, net.table), tokens, x, scale=net.scale)
    ops.norm.artopk_layernorm_forward(x, net.view(weights, net.gamma), net.view(weights, net.beta), y, mean, rstd)
    hidden = torch.relu(y @ net.view(weights, net.w1).t())
    return x, y, mean, rstd, hidden, hidden @ net.view(weights, net.w2).t()


def worker_gradient(net, ops, weights, grad, tokens, targets, first: bool):
    """Adds a micro-batch's gradient to `grad` (overwrites it with `first`); the mean of -log p - entropy_weight entropy."""
    rows = tokens.shape[0]
    x, y, mean, rstd, hidden, logits = forward(net, ops, weights, tokens)
    logp, peak, logsum, entropy = (torch.empty(rows, device=x.device) for _ in range(4))
    ops.tokens.artopk_token_logprobs(logits, targets, logp, peak, logsum, entropy)
    dlogp, dentropy = torch.full_like(logp, -1.0 / rows), torch.full_like(logp, -net.entropy_weight / rows)
    dlogits = logits  # the gradient takes the logits' place
    ops.tokens.artopk_token_logprobs_backward(logits, targets, peak, logsum, dlogits, dlogp=dlogp, entropy=entropy,
                                              dentropy=dentropy)
    dhidden = (dlogits @ net.view(weights, net.w2)) * (hidden > 0)
    dy, dx = dhidden @ net.view(weights, net.w1), torch.empty_like(x)
    ops.norm.artopk_layernorm_backward(dy, x, net.view(weights, net.gamma), mean, rstd, dx, net.view(grad, net.gamma),
                                       net.view(grad, net.beta), accumulate=not first)
    ops.tokens.artopk_embedding_backward(dx, tokens, net.view(grad, net.table), scale=net.scale, accumulate=not first)
    for place, g in ((net.w1, dhidden.t() @ y), (net.w2, dlogits.t() @ hidden)):
        view = net.view(grad, place)
        view.copy_(g) if first else view.add_(g)
    return -(logp.sum() + net.entropy_weight * entropy.sum()) / rows


def initial_weights(net, gen):
    weights = torch.zeros(net.n, device="cuda")
    net.view(weights, net.table).normal_(0.0, 1.0 / math.sqrt(net.width), generator=gen)
    net.view(weights, net.w1).normal_(0.0, 1.0 / math.sqrt(net.width), generator=gen)
    net.view(weights, net.w2).normal_(0.0, 1.0 / math.sqrt(net.hidden), generator=gen)
    net.view(weights, net.gamma).fill_(1.0)
    return weights


def train(steps: int = 60, workers: int = 4, batch: int = 256, micro: int = 2, vocab: int = 200, width: int = 64, hidden: int = 128,
          keep: float = 0.2, eta: float = 0.02, eta_adamw: float = 0.01, seed: int = 0, state_bits: int = 8, keep_weights=None):
    """Losses of the steps, mean over the workers; with `keep_weights` (a list) the network and its weights are put there."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    net = Network(vocab, width, hidden)
    follows = torch.randint(0, vocab, (vocab, 4), generator=gen, device=dev)  # four tokens may follow each
    weights = initial_weights(net, gen)
    grads = [torch.zeros(net.n, device=dev) for _ in range(workers)]
    residuals = [torch.zeros(net.n, device=dev) for _ in range(workers)]
    update, momentum = torch.zeros(net.n, device=dev), torch.zeros(net.n, device=dev)
    seg_k = [math.ceil(keep * (b - a)) for a, b in zip(net.bounds, net.bounds[1:])]
    k = sum(seg_k)
    idx, summed = torch.zeros(k, dtype=torch.int32, device=dev), torch.zeros(k, device=dev)
    ops = Operators(net, batch)
    exchange = artopk.Context(workers, net.n, k, len(seg_k))
    muon = artopk.MatrixContext(net.matrices(), net.n)
    adamw = artopk.AdamWContext(net.tensors(), net.n, state_bits=state_bits)
    moments = adamw.new_state()
    share = 1.0 / (workers * micro)
    losses = []
    for step in range(1, steps + 1):
        total = torch.zeros((), device=dev)
        for g in grads:
            for m in range(micro):
                tokens = torch.randint(0, vocab, (batch,), generator=gen, device=dev)
                pick = torch.randint(0, 4, (batch, 1), generator=gen, device=dev)
                total += worker_gradient(net, ops, weights, g, tokens, follows[tokens].gather(1, pick).view(-1), m == 0)
        exchange.artopk_step(grads, residuals, k, artopk.ARTOPK_STAR, step, idx, summed, update, seg_off=net.bounds, seg_k=seg_k)
        muon.artopk_muon_step(weights, momentum, update, eta=eta, mu=0.9, eta_rest=0.0, update_scale=share)
        adamw.artopk_adamw_step(weights, update, *moments, step=step, eta=eta_adamw, beta2=0.99, update_scale=share, seed=seed)
        losses.append(total * share)
    exchange.status()
    ops.tokens.status()
    if keep_weights is not None:
        keep_weights += [net, weights]
    return [float(v) for v in losses]


def answer(net, weights, first: int, length: int, top: int = 4):
    """The most likely next token `length` times, and each time the `top` most likely with their log probabilities."""
    dev = weights.device
    ops = Operators(net, 1)
    token = torch.tensor([first], dtype=torch.int32, device=dev)
    chosen, alternatives = [], []
    for _ in range(length):
        logits = forward(net, ops, weights, token)[-1]
        ids, logps = torch.empty(1, top, dtype=torch.int32, device=dev), torch.empty(1, top, device=dev)
        ops.tokens.artopk_token_logprobs(logits, top_ids_out=ids, top_logp_out=logps)
        token = ids[:, 0].clone()
        chosen.append(int(token))
        alternatives.append((ids.view(-1).tolist(), logps.view(-1).tolist()))
    return chosen, alternatives


if __name__ == "__main__":
    kept = []
    history = train(keep_weights=kept)
    for i in range(0, len(history), 10):
        print(f"step {i + 1:3d}  loss {history[i]:.4f}")
    print(f"step {len(history):3d}  loss {history[-1]:.4f}  (four equally likely tokens: {math.log(4.0):.4f})")
    tokens, others = answer(*kept, first=0, length=5)
    print("answer", tokens, " alternatives of the first", [f"{t}: {p:.2f}" for t, p in zip(*others[0])])
