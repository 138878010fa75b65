"""Both ends of a language model's training step, and its optimiser beside the matrices, as cases that can be timed and compared.

Five operators: embedding lookup and its gradient (which lands in a worker's flat gradient vector), log probabilities
of given tokens with entropy and top alternatives and their gradient, and an AdamW step over many tensors of a flat
vector with moments in 32 or 8 bits.  listed() names the cases, draw() gives more of the same ranges.  With `own` false
run() computes the definitions with elementary torch operations; with it true it calls the library.
"""

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ETA, BETA1, BETA2, ADAM_EPS, UPDATE_SCALE = 1e-3, 0.9, 0.999, 1e-8, 0.25
#: Elements of a tensor that share the exponents of their 8-bit moments.
BLOCK = 256


def listed():
    def embed(name, call, tokens, vocab, width, table, t, pad=0, accumulate=False, scale=1.0):
        return {"name": name, "call": call, "tokens": tokens, "vocab": vocab, "width": width, "table": table, "type": t,
                "pad": pad, "accumulate": accumulate, "scale": scale}

    def logp(name, call, rows, vocab, t, top=0, pad=0, masked=0.0, scale=1.0):
        return {"name": name, "call": call, "rows": rows, "vocab": vocab, "type": t, "top": top, "pad": pad, "masked": masked,
                "scale": scale}

    def adamw(name, layout, t, bits, loose=0, step=100):
        return {"name": name, "call": "adamw", "layout": layout, "type": t, "bits": bits, "loose": loose, "step": step}

    return [
        # Eight tokens being answered at once: latency.
        embed("embed-8-tokens", "embed", 8, 32000, 4096, "bf16", "bf16"),
        # A large training batch: weights kept in float32, activations in bfloat16, the usual square root as scale.
        embed("embed-32k-mixed", "embed", 32768, 50021, 4096, "f32", "bf16", scale=64.0),
        # A small network's second micro-batch: odd rows at a padded distance, added to the first one's gradient.
        embed("embed-grad-odd-added", "embed_grad", 4099, 9973, 1111, "f32", "f32", pad=3, accumulate=True),
        # A large batch's gradient, the whole table overwritten.
        embed("embed-grad-32k", "embed_grad", 32768, 64000, 2048, "f32", "bf16", scale=0.5),
        # Four tokens being answered, the log probabilities of twenty alternatives shown.
        logp("logp-4-rows-top", "logp", 4, 128000, "bf16", top=20),
        # An evaluation in float32 of a vocabulary of odd size, part of it ruled out.
        logp("logp-odd-f32-top", "logp", 1023, 32003, "f32", top=5, pad=2, masked=0.2),
        # The loss of a large batch.
        logp("logp-16k-rows", "logp", 16384, 64000, "bf16"),
        # Gradient of log probabilities and entropy, half precision, odd rows, a temperature.
        logp("logp-grad-odd-f16", "logp_grad", 2047, 10007, "f16", masked=0.1, scale=0.7),
        # The gradient of the loss over a large vocabulary.
        logp("logp-grad-8k-rows", "logp_grad", 8192, 128000, "bf16"),
        # Gains and biases of a network of some blocks, with a small table: many short tensors.
        adamw("adamw-many-small", "512*120+1536*40+2048*40+511*30+32000+1*20+262144*4", "f32", 32, loose=640),
        # The ResNet50-sized vector as a few long tensors.
        adamw("adamw-25m", "2048000+9437184+4718592+9353256", "f32", 32),
        # An embedding and a head kept in bfloat16, moments in 8 bits.
        adamw("adamw-131m-8bit", "65536000+65536000+2048*8", "bf16", 8, loose=1),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    call = rng.choice(["embed", "embed_grad", "embed_grad", "logp", "logp", "logp_grad", "adamw", "adamw"])
    t = rng.choice(["f32", "bf16", "f16"])
    pad = rng.choice([0, 0, 1, 8])
    if call.startswith("embed"):
        width = rng.choice([_log_int(rng, 1, 8192), 64 * _log_int(rng, 1, 128)])
        return {"call": call, "tokens": _log_int(rng, 1, min(131072, 134217728 // width)),
                "vocab": _log_int(rng, 16, min(131072, 268435456 // width)), "width": width,
                "table": rng.choice(["f32", "bf16", "f16"]), "type": t, "pad": pad,
                "accumulate": call == "embed_grad" and rng.random() < 0.5, "scale": rng.choice([1.0, 0.37, 16.0])}
    if call.startswith("logp"):
        vocab = rng.choice([_log_int(rng, 2, 200000), 64 * _log_int(rng, 1, 3000)])
        most = (400000000 if t == "f32" else 800000000) // (vocab + 8)
        return {"call": call, "rows": _log_int(rng, 1, min(32768, most)), "vocab": vocab, "type": t,
                "top": min(vocab, rng.choice([0, 0, 1, 5, 20, 32])) if call == "logp" else 0, "pad": pad,
                "masked": rng.choice([0.0, 0.0, 0.3]), "scale": rng.choice([1.0, 1.0, 0.5, 1.4])}
    parts, left = [], 1 << 27
    for _ in range(rng.choice([1, 2, 4, 7])):
        count, reps = _log_int(rng, 1, 1 << 26), rng.choice([1, 1, 2, 9, 50])
        if count * reps <= left:
            parts.append("%d*%d" % (count, reps))
            left -= count * reps
    return {"call": call, "layout": "+".join(parts or ["4097*3"]), "type": t, "bits": rng.choice([32, 8, 8]),
            "loose": rng.choice([0, 1, 64, 1000]), "step": _log_int(rng, 1, 100000)}


# ---- inputs ------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rows(rows, cols, pad, t, values=None):
    """Rows `pad` elements further apart than they are long."""
    kept = torch.zeros(rows, cols + pad, dtype=t, device="cuda")
    if values is not None:
        kept[:, :cols] = values
    return kept[:, :cols]


def _tokens(g, count, vocab):
    """Low numbers more often than high ones, as in text, and one place in fifty that holds no token."""
    u = torch.rand(count, generator=g, device="cuda", dtype=torch.float64)
    tok = (torch.exp(u * math.log(vocab + 1.0)) - 1.0).long().clamp_(0, vocab - 1)
    none = torch.rand(count, generator=g, device="cuda") < 0.02
    return torch.where(none, torch.full_like(tok, -1), tok)


def _distinct(count, vocab):
    """How many different tokens _tokens() is expected to give."""
    v = np.arange(vocab, dtype=np.float64)
    p = np.log((v + 2.0) / (v + 1.0)) / math.log(vocab + 1.0)
    return float(np.sum(1.0 - np.exp(count * np.log1p(-np.minimum(p, 1.0 - 1e-12)))))


def _embed_inputs(case, seed):
    g, t = _gen(seed), TYPES[case["type"]]
    s = {"tokens": _tokens(g, case["tokens"], case["vocab"])}
    if case["call"] == "embed":
        s["table"] = (0.02 * _randn(g, case["vocab"], case["width"])).to(TYPES[case["table"]])
    else:
        s["dy"] = _rows(case["tokens"], case["width"], case["pad"], t, 0.1 * _randn(g, case["tokens"], case["width"]))
        s["dtable"] = (0.1 * _randn(g, case["vocab"], case["width"])).to(TYPES[case["table"]])
    return s


def _logp_inputs(case, seed):
    """Logits of which some stand out, as a trained model's do; every thirtieth row of a masked case has nothing left."""
    g, rows, vocab = _gen(seed), case["rows"], case["vocab"]
    z = _randn(g, rows, vocab).mul_(1.5)
    hot = torch.randint(0, vocab, (rows, 4), generator=g, device="cuda")
    z.scatter_add_(1, hot, 6.0 + 3.0 * _randn(g, rows, 4))
    if case["masked"]:
        z.masked_fill_(torch.rand(rows, vocab, generator=g, device="cuda") < case["masked"], -math.inf)
        z[29::30] = -math.inf
    s = {"logits": _rows(rows, vocab, case["pad"], TYPES[case["type"]], z)}
    tok = _tokens(g, rows, vocab)
    s["tokens"] = torch.where((tok >= 0) & (torch.rand(rows, generator=g, device="cuda") < 0.5), hot[:, 0], tok)
    del z
    if case["call"] == "logp_grad":
        s["peak"], logsum, entropy = _row_sums(s["logits"], case["scale"])
        s["logsum"], s["entropy"] = logsum.float(), entropy.float()
        mean = 1.0 if case["type"] == "f16" else 1.0 / rows  # (half precision: of a loss that is scaled by the rows)
        s["dlogp"] = -mean * (0.5 + torch.rand(rows, generator=g, device="cuda"))
        s["dlse"] = 1e-3 * mean * torch.rand(rows, generator=g, device="cuda")
        s["dentropy"] = 0.1 * mean * _randn(g, rows)
    return s


def _row_sums(logits, scale):
    """Statistics that the forward pass left: the largest logit, and the logarithm of the sum relative to it and the entropy
    in 64 bits, some rows at a time."""
    peak = logits.float().amax(1)
    logsum = torch.empty(logits.shape[0], dtype=torch.float64, device="cuda")
    entropy = torch.empty_like(logsum)
    some = max(1, 100000000 // logits.shape[1])
    for at in range(0, logits.shape[0], some):
        top = peak[at:at + some].double().view(-1, 1)
        none = top.view(-1) == -math.inf
        d = logits[at:at + some].double().sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).mul_(float(np.float32(scale)))
        e = torch.exp(d)
        total = e.sum(1)
        weighted = e.mul_(d.clamp_(min=-1e30)).sum(1)
        logsum[at:at + some] = torch.where(none, 0.0, torch.log(total))
        entropy[at:at + some] = torch.where(none, 0.0, torch.log(total) - weighted / total)
    return peak, logsum, entropy


def _tensors(case):
    """([(offset, count, factor of eta, decay)], elements of the flat vector); `loose` elements follow every tensor."""
    at, out = 0, []
    for part in case["layout"].split("+"):
        count, _, reps = part.partition("*")
        for _ in range(int(reps or 1)):
            out.append((at, int(count), 1.0 if len(out) % 3 else 0.5, 0.1 if int(count) >= 4096 else 0.0))
            at += int(count) + case["loose"]
    return out, at


def _places(tensors):
    """For each element of the moments its place in the flat vector, -1 where a tensor's last block is not full; and factor
    of eta and decay of each block."""
    parts, eta, decay = [], [], []
    for at, count, factor, dec in tensors:
        blocks = -(-count // BLOCK)
        p = torch.arange(at, at + blocks * BLOCK, dtype=torch.int64, device="cuda")
        p[count:] = -1
        parts.append(p)
        eta += [torch.full((blocks, 1), factor, device="cuda")]
        decay += [torch.full((blocks, 1), dec, device="cuda")]
    return torch.cat(parts), torch.cat(eta), torch.cat(decay)


def _adamw_inputs(case, seed):
    g = _gen(seed)
    tensors, n = _tensors(case)
    place, eta, decay = _places(tensors)
    size = torch.exp(_randn(g, n))  # elements' gradients differ in size
    update = 4e-3 * size * _randn(g, n)
    s = {"update": update, "weights": (0.02 * _randn(g, n)).to(TYPES[case["type"]]), "place": place, "eta": eta, "decay": decay}
    held = place.clamp(min=0)
    m = torch.where(place >= 0, (3e-4 * size * _randn(g, n))[held], torch.zeros((), device="cuda"))
    v = torch.where(place >= 0, ((1e-3 * size) ** 2 * (0.5 + torch.rand(n, generator=g, device="cuda")))[held],
                    torch.zeros((), device="cuda"))
    if case["bits"] == 8:
        half = torch.full((place.numel(),), 1 << 19, dtype=torch.int32, device="cuda")
        s["first"], e1 = _encode_first(m.view(-1, BLOCK), half.view(-1, BLOCK))
        s["second"], e2 = _encode_second(v.view(-1, BLOCK), half.view(-1, BLOCK))
        s["first"], s["second"] = s["first"].view(-1), s["second"].view(-1)
        s["scales"] = torch.cat([e1, e2], 1).contiguous()
        s["seed"] = seed & 0xFFFF
    else:
        s["first"], s["second"], s["scales"] = m, v, None
    return s


def _plan(case):
    """The handle that a program keeps between steps."""
    if not own:
        return None
    import paper_2312_02493_amd as artopk

    if case["call"] == "adamw":
        tensors, n = _tensors(case)
        return artopk.AdamWContext(tensors, n, {"f32": artopk.ARTOPK_G_F32, "bf16": artopk.ARTOPK_G_BF16,
                                                "f16": artopk.ARTOPK_G_F16}[case["type"]], case["bits"])
    if case["call"].startswith("embed"):
        return artopk.TokenContext(case["tokens"], case["vocab"], case["width"])
    return artopk.TokenContext(case["rows"], case["vocab"])


def prepare(case, seed):
    s = {"case": case, "plan": _plan(case)}
    if case["call"] == "adamw":
        s.update(_adamw_inputs(case, seed))
        if case["bits"] == 8:
            s["values"] = [torch.zeros(s["first"].numel(), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    elif case["call"].startswith("embed"):
        s.update(_embed_inputs(case, seed))
        if case["call"] == "embed":
            s["y"] = _rows(case["tokens"], case["width"], case["pad"], TYPES[case["type"]])
    else:
        s.update(_logp_inputs(case, seed))
        if case["call"] == "logp":
            rows, top = case["rows"], case["top"]
            s["logp"], s["peak"], s["logsum"], s["entropy"] = (torch.zeros(rows, device="cuda") for _ in range(4))
            s["top_ids"] = torch.zeros(rows, top, dtype=torch.int32, device="cuda") if top else None
            s["top_logp"] = torch.zeros(rows, top, device="cuda") if top else None
        else:
            s["dlogits"] = _rows(case["rows"], case["vocab"], case["pad"], TYPES[case["type"]])
    return s


# ---- moments in 8 bits -------------------------------------------------------------------------
# A block's elements share the largest exponent field E among them (one byte).  A code is an exponent field and three bits of
# mantissa: 2^(field - top + E - 127) (1 + mantissa / 8), multiples of the same step below field 1; `top` is 14 for the first
# moment, whose code has a sign before it, and 30 for the second.  Rounding is up with the probability of the part cut off.
TOP1, TOP2 = 14, 30


def _exponents(x, least):
    """E of each block of [blocks, BLOCK], at least `least`; 255 where there is infinity or NaN."""
    return ((x.view(torch.int32) >> 23) & 255).amax(1, keepdim=True).clamp(min=least)


def _encode_first(m, rnd):
    e = _exponents(m, TOP1 + 1)
    mag = m.abs()
    t = mag.view(torch.int32) - ((e - TOP1) << 23)
    step = torch.ldexp(mag, 64 + torch.zeros_like(e))  # two factors: one would be beyond float32
    step = step * _pow2()[(127 + TOP1 + 2 - 64 + 127 - e).clamp(0, 254).long()]
    low = torch.floor(step + rnd.float() * 2.0 ** -20).clamp(max=8.0).int()
    code = torch.where(t >= 1 << 23, (t + rnd) >> 20, low)
    code = torch.where(m.view(torch.int32) < 0, code | 128, code)
    return code.to(torch.uint8), e.to(torch.uint8)


def _encode_second(v, rnd):
    e = _exponents(v, TOP2 + 1)
    bits = v.view(torch.int32)
    t = bits - ((e - TOP2) << 23)
    code = torch.where(t >= 1 << 23, (t + rnd) >> 20, torch.where(bits != 0, 8, 0).int())
    return code.to(torch.uint8), e.to(torch.uint8)


_kept = {}


def _pow2():
    """2^(i - 127) for the exponent fields i."""
    if "pow2" not in _kept:
        _kept["pow2"] = torch.tensor(2.0 ** (np.arange(256.0) - 127.0), dtype=torch.float32, device="cuda")
    return _kept["pow2"]


def _code_values(sign, top):
    if top not in _kept:
        code = np.arange(256)
        field, man = (code & 127) >> 3 if sign else code >> 3, code & 7
        v = np.where(field > 0, 2.0 ** (field - top) * (1 + man / 8), 2.0 ** (1 - top) * man / 8)
        if sign:
            v = np.where(code & 128, -v, v)
        _kept[top] = torch.tensor(v, dtype=torch.float32, device="cuda")
    return _kept[top]


def _decode(code, e, sign, top):
    v = _code_values(sign, top)[code.long()] * _pow2()[e.long()]
    return torch.where(e == 255, torch.full_like(v, math.nan), v)


def _random_bits(count, seed, step):
    """32 bits for each place of the moments, from the seed and the step."""
    wide = (seed + step * 0x9E3779B97F4A7C15) & 0xFFFFFFFFFFFFFFFF
    key = (wide ^ (wide >> 32)) & 0xFFFFFFFF
    x = torch.arange(count, dtype=torch.int64, device="cuda")
    x = (x * 0x9E3779B1 + key) & 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x6A09E667) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


# ---- one pass ----------------------------------------------------------------------------------
def _plain_embed(s):
    case, tok = s["case"], s["tokens"]
    if case["call"] == "embed":
        rows = s["table"][tok.clamp(min=0)].float() * case["scale"]
        s["y"].copy_(torch.where(tok.view(-1, 1) >= 0, rows, torch.zeros((), device="cuda")))
        return {"y": s["y"]}
    held = torch.where(tok >= 0, tok, torch.full_like(tok, case["vocab"]))  # (no token: a row that is dropped)
    total = torch.zeros(case["vocab"] + 1, case["width"], device="cuda")
    total.index_add_(0, held, s["dy"].float())
    total = total[:-1] * case["scale"]
    s["dtable"].copy_(s["dtable"].float() + total if case["accumulate"] else total)
    return {"dtable": s["dtable"]}


def _plain_logp(s):
    case, tok, scale = s["case"], s["tokens"], s["case"]["scale"]
    x = s["logits"].float()
    zero = torch.zeros((), device="cuda")
    at = tok.clamp(min=0).view(-1, 1)
    if case["call"] == "logp":
        # the largest element's own 1 stays out of the sum: a sure answer's logarithm lies close to zero
        top, where = x.max(1, keepdim=True)
        none = top == -math.inf
        d = (x - torch.where(none, zero, top)) * scale
        e = torch.exp(d).scatter_(1, where, 0.0)
        rest = e.sum(1)
        log = torch.log1p(rest)
        base = torch.where(none.view(-1), zero, log).view(-1, 1)
        logp = torch.where(tok >= 0, (d.gather(1, at) - base).view(-1), zero)
        weighted = torch.where(e > 0, e * d, zero).sum(1)
        out = {"logp": logp, "peak": top.view(-1), "logsum": base.view(-1),
               "entropy": torch.where(none.view(-1), zero, log - weighted / (1.0 + rest))}
        if case["top"]:
            bits = (x + 0.0).view(torch.int32)
            order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32
            order = order + (0x7FFFFFFF - torch.arange(case["vocab"], device="cuda"))
            ids = 0x7FFFFFFF - (torch.topk(order, case["top"], 1).values & 0xFFFFFFFF)
            out["top_ids"], out["top_logp"] = ids.int(), d.gather(1, ids) - base
        return out
    none = s["peak"].view(-1, 1) == -math.inf
    top, logsum, dent = torch.where(none, zero, s["peak"].view(-1, 1)), s["logsum"].view(-1, 1), s["dentropy"].view(-1, 1)
    dlogp, h = torch.where(tok >= 0, s["dlogp"], zero).view(-1, 1), s["entropy"].view(-1, 1)
    d = (x - top) * scale - logsum
    p = torch.exp(d)
    grad = p * (s["dlse"].view(-1, 1) - dlogp) - dent * torch.where(p > 0, p * (d + h), zero)
    # at the token itself 1 - p, from 64 bits where p is close to 1
    d = (x.gather(1, at).double() - top) * scale - logsum
    p = torch.exp(d)
    own_ = -dlogp * torch.expm1(d) + s["dlse"].view(-1, 1) * p - dent * torch.where(p > 0, p * (d + h), 0.0)
    grad.scatter_(1, at, own_.float())
    s["dlogits"].copy_(torch.where(none, zero, grad * scale))
    return {"dlogits": s["dlogits"]}


def _plain_adamw(s):
    case, place, w = s["case"], s["place"], s["weights"]
    held = place >= 0
    at = place.clamp(min=0)
    zero = torch.zeros((), device="cuda")
    g = torch.where(held, UPDATE_SCALE * s["update"][at], zero).view(-1, BLOCK)
    m, v = s["first"].view(-1, BLOCK), s["second"].view(-1, BLOCK)
    if case["bits"] == 8:
        m = _decode(m, s["scales"][:, :1], True, TOP1)
        v = _decode(v, s["scales"][:, 1:], False, TOP2)
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    step = case["step"]
    root = torch.sqrt(v) * (1.0 / math.sqrt(1.0 - BETA2 ** step)) + ADAM_EPS
    x = w[at].float().view(-1, BLOCK)
    x = x * (1.0 - ETA * s["eta"] * s["decay"]) - (ETA / (1.0 - BETA1 ** step)) * s["eta"] * (m / root)
    w[place[held]] = x.view(-1)[held].to(w.dtype)
    if case["bits"] == 32:
        s["first"].copy_(m.view(-1))
        s["second"].copy_(v.view(-1))
        return {"weights": w, "first": s["first"], "second": s["second"]}
    r = _random_bits(place.numel(), s["seed"], step).view(-1, BLOCK)
    first, e1 = _encode_first(m, (((r & 0xFFFF) << 4) | 8).int())
    second, e2 = _encode_second(v, (((r >> 16) << 4) | 8).int())
    s["first"].copy_(first.view(-1))
    s["second"].copy_(second.view(-1))
    s["scales"].copy_(torch.cat([e1, e2], 1))
    s["values"][0].copy_(_decode(first, e1, True, TOP1).view(-1))
    s["values"][1].copy_(_decode(second, e2, False, TOP2).view(-1))
    return {"weights": w, "first": s["values"][0], "second": s["values"][1]}


def _plain(s):
    call = s["case"]["call"]
    return _plain_adamw(s) if call == "adamw" else _plain_embed(s) if call.startswith("embed") else _plain_logp(s)


def run(s):
    if not own:
        return _plain(s)
    case, plan = s["case"], s["plan"]
    if case["call"] == "embed":
        plan.artopk_embedding_forward(s["table"], s["tokens"], s["y"], scale=case["scale"])
        return {"y": s["y"]}
    if case["call"] == "embed_grad":
        plan.artopk_embedding_backward(s["dy"], s["tokens"], s["dtable"], scale=case["scale"], accumulate=case["accumulate"])
        return {"dtable": s["dtable"]}
    if case["call"] == "logp":
        plan.artopk_token_logprobs(s["logits"], s["tokens"], s["logp"], s["peak"], s["logsum"], s["entropy"], s["top_ids"],
                                   s["top_logp"], scale=case["scale"])
        out = {"logp": s["logp"], "peak": s["peak"], "logsum": s["logsum"], "entropy": s["entropy"]}
        return {**out, "top_ids": s["top_ids"], "top_logp": s["top_logp"]} if case["top"] else out
    if case["call"] == "logp_grad":
        plan.artopk_token_logprobs_backward(s["logits"], s["tokens"], s["peak"], s["logsum"], s["dlogits"], dlogp=s["dlogp"],
                                            dlse=s["dlse"], entropy=s["entropy"], dentropy=s["dentropy"], scale=case["scale"])
        return {"dlogits": s["dlogits"]}
    plan.artopk_adamw_step(s["weights"], s["update"], s["first"], s["second"], s["scales"], step=case["step"], eta=ETA,
                           beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, update_scale=UPDATE_SCALE, seed=s.get("seed", 0))
    if case["bits"] == 32:
        return {"weights": s["weights"], "first": s["first"], "second": s["second"]}
    plan.artopk_adamw_values(s["first"], s["second"], s["scales"], *s["values"])
    return {"weights": s["weights"], "first": s["values"][0], "second": s["values"][1]}


def _size(t):
    return 4 if t == "f32" else 2


def work(case):
    if case["call"].startswith("embed"):
        rows, width = case["tokens"], case["width"]
        some = _distinct(rows, case["vocab"]) * width * _size(case["table"])
        moved = rows * width * _size(case["type"]) + 8 * rows
        if case["call"] == "embed":
            return {"bytes": moved + some, "flops": rows * width}
        whole = case["vocab"] * width * _size(case["table"])
        return {"bytes": moved + (2 * some if case["accumulate"] else whole), "flops": 2 * rows * width}
    if case["call"].startswith("logp"):
        rows, elems = case["rows"], case["rows"] * case["vocab"]
        if case["call"] == "logp":
            return {"bytes": elems * _size(case["type"]) + rows * (24 + 8 * case["top"]), "flops": 8 * elems}
        return {"bytes": 2 * elems * _size(case["type"]) + 32 * rows, "flops": 10 * elems}
    n = sum(count for _, count, _, _ in _tensors(case)[0])
    moved = 2 * _size(case["type"]) + 4 + (16 if case["bits"] == 32 else 4 + 4 / BLOCK + 4)  # (8 bits: and their values)
    return {"bytes": moved * n, "flops": (15 if case["bits"] == 32 else 40) * n}


# ---- the definitions in 64 bits ----------------------------------------------------------------
def _exact_embed(case, seed):
    s = _embed_inputs(case, seed)
    tok, scale = s["tokens"], float(np.float32(case["scale"]))
    live = torch.nonzero(tok >= 0).view(-1)
    if case["call"] == "embed":
        y = torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device="cuda")
        y[live] = torch.index_select(s["table"], 0, tok[live]).double() * scale
        return {"y": y}
    grad = s["dtable"].double() if case["accumulate"] else torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda")
    # the tokens' rows side by side: differences of running sums where a token ends
    by = torch.argsort(tok[live], stable=True)
    names, counts = torch.unique_consecutive(tok[live][by], return_counts=True)
    ends = torch.cumsum(counts, 0)
    some = max(1, 100000000 // max(1, live.numel()))
    for c in range(0, case["width"], some):
        run_ = torch.cumsum(s["dy"][live][by, c:c + some].double(), 0)[ends - 1]
        run_[1:] -= run_[:-1].clone()
        grad[names, c:c + some] += scale * run_
    return {"dtable": grad}


def _exact_logp(case, seed):
    s = _logp_inputs(case, seed)
    tok, x, scale = s["tokens"], s["logits"], float(np.float32(case["scale"]))
    row = torch.arange(case["rows"], device="cuda")
    if case["call"] == "logp":
        peak, logsum, entropy = _row_sums(x, scale)
        base = logsum + torch.nan_to_num(peak.double(), neginf=0.0) * scale
        logp = torch.where(tok >= 0, x[row, tok.clamp(min=0)].double() * scale - base, 0.0)
        out = {"logp": logp, "peak": peak, "logsum": logsum, "entropy": entropy}
        if case["top"]:
            k = case["top"]
            out["top_ids"] = None
            out["top_logp"] = torch.topk(x.float(), k, 1).values.double() * scale - base.view(-1, 1)
        return out
    out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
    some = max(1, 100000000 // case["vocab"])
    for at in range(0, case["rows"], some):
        cut = slice(at, at + some)
        lse, h = s["peak"][cut].double().view(-1, 1) * scale + s["logsum"][cut].double().view(-1, 1), s["entropy"][cut].double().view(-1, 1)
        dead = lse == -math.inf
        dlse = s["dlse"][cut].double().view(-1, 1)
        lp = (x[cut].double() * scale - lse.masked_fill(dead, 0.0)).clamp(min=-1e4)  # (e^-1e4 is 0 in 64 bits)
        one = torch.zeros_like(lp)
        live = torch.nonzero(tok[cut] >= 0).view(-1)
        one[live, tok[cut][live]] = 1.0
        dlogp = torch.zeros_like(dlse)
        dlogp[live] = s["dlogp"][cut].double().view(-1, 1)[live]
        p = torch.exp(lp)
        grad = dlogp * (one - p) + dlse * p - s["dentropy"][cut].double().view(-1, 1) * p * (lp + h)
        out[cut] = (grad * scale).masked_fill(dead, 0.0)
    return {"dlogits": out}


def _exact_adamw(case, seed):
    s = _adamw_inputs(case, seed)
    tensors, _ = _tensors(case)
    w, u = s["weights"].double(), s["update"].double() * UPDATE_SCALE
    first, second = s["first"].double(), s["second"].double()
    if case["bits"] == 8:
        first = _decode(s["first"].view(-1, BLOCK), s["scales"][:, :1], True, TOP1).double().view(-1)
        second = _decode(s["second"].view(-1, BLOCK), s["scales"][:, 1:], False, TOP2).double().view(-1)
    b1, b2 = float(BETA1), float(BETA2)
    at = 0
    for offset, count, factor, decay in tensors:
        blocks = -(-count // BLOCK)
        g = u[offset:offset + count]
        m = first[at:at + count].mul_(b1).add_(g, alpha=1.0 - b1)
        v = second[at:at + count].mul_(b2).addcmul_(g, g, value=1.0 - b2)
        way = (m / (1.0 - b1 ** case["step"])) / (torch.sqrt(v / (1.0 - b2 ** case["step"])) + ADAM_EPS)
        eta = ETA * factor
        w[offset:offset + count] = (1.0 - eta * decay) * w[offset:offset + count] - eta * way
        at += blocks * BLOCK
    if case["bits"] == 8:
        r = _random_bits(at, s["seed"], case["step"]).double()
        high = torch.floor(r / 65536.0)
        for x, u16, low, top in ((first, r - 65536.0 * high, 14, TOP1), (second, high, 30, TOP2)):
            x = x.view(-1, BLOCK)
            mag = x.abs()
            field = torch.frexp(mag)[1] - 1  # of 1 <= significand < 2
            field = torch.where(mag > 0, field, torch.full_like(field, -1000))
            most = field.amax(1, keepdim=True).clamp(min=top + 1 - 127)
            step = torch.pow(2.0, (torch.maximum(field, most - (top - 1)) - 3).double())
            q = torch.floor(mag / step + (u16.view(-1, BLOCK) * 16.0 + 8.0) / 1048576.0) * step
            if top == TOP2:
                least = torch.pow(2.0, (most - (top - 1)).double())
                q = torch.where((mag > 0) & (mag < least), least.expand_as(q), q)
            x.copy_(torch.where(x < 0, -q, q))
    return {"weights": w, "first": first, "second": second}


def exact(case, seed):
    if case["call"] == "adamw":
        return _exact_adamw(case, seed)
    return _exact_embed(case, seed) if case["call"].startswith("embed") else _exact_logp(case, seed)
