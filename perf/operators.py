"""What a training step does before and after the compressed exchange, as cases that can be timed and compared.

Four operators: layer norm forward, layer norm backward (whose weight gradients land in a worker's flat
gradient vector), the orthogonalisation of update matrices that lie in a flat vector, and the step that
takes the exchanged dense update through momentum and orthogonalisation to the weights.  listed() names
the cases, draw() gives more of the same ranges.  With `own` false run() computes the definitions with
elementary torch operations in float32; with it true it calls the library.
"""

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
#: Coefficients (a, b, c) of one odd polynomial step p(s) = a s + b s^3 + c s^5 on the singular values.
STEP = (3.4445, -4.7750, 2.0315)
STEPS = 5
NORM_EPS = 1e-7
LN_EPS = 1e-5
ETA, MU, DECAY, ETA_REST = 0.02, 0.95, 0.01, 0.005


# ---- layouts of matrices in a flat vector: "RxC*COUNT" joined by "+", and loose elements behind each matrix --
def _network_11m():
    """Convolutions as matrices (channels out x channels in times window) of a small image network."""
    parts = ["64x147", "64x576*4", "128x576", "128x1152*3", "128x64", "256x1152", "256x2304*3", "256x128", "512x2304",
             "512x4608*3", "512x256", "1000x512"]
    return "+".join(parts)


def _matrices(case):
    """([(offset, rows, cols)], elements of the flat vector); `loose` elements (a bias, gains) follow every matrix."""
    at, out = 0, []
    for part in case["layout"].split("+"):
        size, _, count = part.partition("*")
        r, c = (int(v) for v in size.split("x"))
        for _ in range(int(count or 1)):
            out.append((at, r, c))
            at += r * c + case.get("loose", 0)
    return out, at


def _scale(r, c):
    return math.sqrt(max(1.0, r / c))


def listed():
    def norm(name, call, rows, cols, t, pad=0, accumulate=False):
        return {"name": name, "call": call, "rows": rows, "cols": cols, "type": t, "pad": pad, "accumulate": accumulate}

    def flat(name, call, layout, t, loose=0, nesterov=True):
        return {"name": name, "call": call, "layout": layout, "type": t, "loose": loose, "nesterov": nesterov}

    return [
        # Eight tokens being answered at once: latency is all there is.
        norm("norm-fwd-8-tokens", "norm_fwd", 8, 4096, "bf16"),
        # Rows of an odd length, one behind the other, so that most begin off any boundary.
        norm("norm-fwd-odd-f32", "norm_fwd", 4099, 1111, "f32"),
        # The activations of a large training batch.
        norm("norm-fwd-32k", "norm_fwd", 32768, 4096, "bf16"),
        # A small network's layer.
        norm("norm-bwd-small", "norm_bwd", 257, 512, "f32"),
        # Odd rows kept at a padded distance, half precision.
        norm("norm-bwd-odd-f16", "norm_bwd", 8191, 2501, "f16", pad=3),
        # A large batch, second micro-batch: gradients are added to what the first left.
        norm("norm-bwd-32k", "norm_bwd", 32768, 2048, "bf16", accumulate=True),
        # One small layer by itself: launches.
        flat("orth-one-small", "orth", "96x160", "f32"),
        # The attention and feed-forward matrices of one block of a middling network, full precision.
        flat("orth-block-f32", "orth", "640x640*4+2560x640+640x2560", "f32"),
        # One large layer of a network kept in bfloat16.
        flat("orth-large-bf16", "orth", "4096x4096", "bf16"),
        # A small classifier with its biases.
        flat("muon-small", "muon", "256x784+128x256+10x128", "f32", loose=64),
        # The ResNet18-sized vector layer by layer, convolutions as matrices, the norms' gains between them.
        flat("muon-11m-convs", "muon", _network_11m(), "f32", loose=128),
        # Four transformer blocks, weights kept in bfloat16.
        flat("muon-78m-blocks", "muon", "+".join(["1280x1280*4+5120x1280+1280x5120"] * 4), "bf16", loose=2560),
    ]


def _log_int(rng, lo, hi):
    v = min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))
    return v + 1 if v == 3072 else v


def draw(rng):
    call = rng.choice(["norm_fwd", "norm_bwd", "orth", "orth", "muon", "muon"])
    t = rng.choice(["f32", "bf16", "f16"])
    if call.startswith("norm"):
        cols = rng.choice([_log_int(rng, 64, 16384), 64 * _log_int(rng, 1, 256) - rng.choice([0, 0, 0, 32])])
        cols += cols == 3072
        most = 134217728 if call == "norm_fwd" else 67108864
        return {"call": call, "rows": _log_int(rng, 1, min(65536, most // (cols + 8))), "cols": cols, "type": t,
                "pad": rng.choice([0, 0, 1, 8]), "accumulate": call == "norm_bwd" and rng.random() < 0.5}
    budget, parts, loose = 3.0e11, [], rng.choice([0, 1, 64, 1000])
    for _ in range(rng.choice([1, 1, 2, 3, 5, 8])):
        r, c, count = _log_int(rng, 16, 4096), _log_int(rng, 16, 4096), rng.choice([1, 1, 1, 2, 4, 7])
        if call == "orth" and t == "f32":  # larger ones amplify float32's own roundings beyond use
            r, c = (min(r, 640), c) if r < c else (r, min(c, 640))
        need = count * _flops(r, c)
        if need <= budget:
            parts.append("%dx%d*%d" % (r, c, count))
            budget -= need
    return {"call": call, "layout": "+".join(parts or ["333x444*2"]), "type": t, "loose": loose,
            "nesterov": rng.random() < 0.7}


def _flops(r, c):
    """Of all steps on one matrix: two symmetric products (half of each is needed) and one full one a step."""
    m, n = min(r, c), max(r, c)
    return STEPS * (m * m * n + m * m * m + 2 * m * m * n)


# ---- inputs ------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _norm_inputs(case, seed):
    g, rows, cols, t = _gen(seed), case["rows"], case["cols"], TYPES[case["type"]]

    def rows_of(make):
        """`make`'s values as rows `pad` elements further apart than they are long."""
        kept = torch.zeros(rows, cols + case["pad"], dtype=t, device="cuda")
        kept[:, :cols] = make
        return kept[:, :cols]

    s = {"x": rows_of(_randn(g, rows, cols) * (0.5 + torch.rand(rows, 1, generator=g, device="cuda"))
                      + _randn(g, rows, 1)),
         "gamma": 1.0 + 0.1 * _randn(g, cols), "beta": 0.1 * _randn(g, cols)}
    if case["call"] == "norm_bwd":
        s["dy"] = rows_of(_randn(g, rows, cols) * 0.1)
        x = s["x"].double()
        mean = x.mean(1, keepdim=True)
        s["rstd"] = ((x - mean).square().mean(1) + LN_EPS).rsqrt().float()
        s["mean"] = mean.view(-1).float()
        s["dgamma"], s["dbeta"] = 0.1 * _randn(g, cols), 0.1 * _randn(g, cols)
    return s


def _flat_inputs(case, seed):
    """The flat vector holds, matrix by matrix, a few strong directions and noise around them, as gradients do."""
    g = _gen(seed)
    mats, n = _matrices(case)
    v = 1e-3 * _randn(g, n)
    for at, r, c in mats:
        k = max(1, min(r, c) // 8)
        v[at:at + r * c] += 1e-3 * (_randn(g, r, k) @ _randn(g, k, c)).view(-1) / math.sqrt(k)
    t = TYPES[case["type"]]
    if case["call"] == "orth":
        return {"x": v.to(t)}
    w = 0.02 * _randn(g, n)
    return {"weights": w.to(t), "momentum": 5.0 * v + 2e-3 * _randn(g, n), "update": v}


def _plan(case):
    """The handle that a program keeps between steps."""
    if not own:
        return None
    import paper_2312_02493_amd as artopk

    if case["call"].startswith("norm"):
        return artopk.NormContext(case["rows"], case["cols"])
    mats, n = _matrices(case)
    return artopk.MatrixContext([(at, r, c, _scale(r, c)) for at, r, c in mats], n,
                                {"f32": artopk.ARTOPK_G_F32, "bf16": artopk.ARTOPK_G_BF16,
                                 "f16": artopk.ARTOPK_G_F16}[case["type"]])


def prepare(case, seed):
    s = {"case": case, "plan": _plan(case)}
    if case["call"].startswith("norm"):
        s.update(_norm_inputs(case, seed))
        s["y" if case["call"] == "norm_fwd" else "dx"] = torch.zeros_like(s["x"])
        if case["call"] == "norm_fwd":
            s["mean"], s["rstd"] = torch.zeros(case["rows"], device="cuda"), torch.zeros(case["rows"], device="cuda")
        return s
    s.update(_flat_inputs(case, seed))
    s["mats"] = _matrices(case)[0]
    if case["call"] == "orth":
        s["out"] = torch.zeros_like(s["x"])
    else:
        inside = torch.zeros(s["weights"].numel(), dtype=torch.bool, device="cuda")
        for at, r, c in s["mats"]:
            inside[at:at + r * c] = True
        s["loose"] = torch.nonzero(~inside).view(-1)  # positions that belong to no matrix
    return s


# ---- one pass ----------------------------------------------------------------------------------
def _orthogonal(x):
    """Steps of the polynomial on x over its Frobenius norm; float32 in and out."""
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.square().sum().sqrt() + NORM_EPS)
    a, b, c = STEP
    for _ in range(STEPS):
        s = x @ x.t()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if tall else x


def _plain(s):
    case = s["case"]
    if case["call"] == "norm_fwd":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = (d.square().mean(1, keepdim=True) + LN_EPS).rsqrt()
        s["y"].copy_(d * rstd * s["gamma"] + s["beta"])
        return {"y": s["y"], "mean": mean.view(-1), "rstd": rstd.view(-1)}
    if case["call"] == "norm_bwd":
        hat = (s["x"].float() - s["mean"].view(-1, 1)) * s["rstd"].view(-1, 1)
        dy = s["dy"].float()
        d = dy * s["gamma"]
        s["dx"].copy_(s["rstd"].view(-1, 1) * (d - d.mean(1, keepdim=True) - hat * (d * hat).mean(1, keepdim=True)))
        dgamma, dbeta = (dy * hat).sum(0), dy.sum(0)
        if case["accumulate"]:
            dgamma, dbeta = s["dgamma"] + dgamma, s["dbeta"] + dbeta
        s["dgamma"].copy_(dgamma)
        s["dbeta"].copy_(dbeta)
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if case["call"] == "orth":
        for at, r, c in s["mats"]:
            o = _orthogonal(s["x"][at:at + r * c].view(r, c).float())
            s["out"][at:at + r * c].view(r, c).copy_(_scale(r, c) * o)
        return {"out": s["out"]}
    w, m, u = s["weights"], s["momentum"], s["update"]
    m.mul_(MU).add_(u)
    v = MU * m + u if case["nesterov"] else m
    for at, r, c in s["mats"]:
        o = _orthogonal(v[at:at + r * c].view(r, c))
        q = w[at:at + r * c].view(r, c)
        q.copy_(q.float() * (1.0 - ETA * DECAY) - ETA * _scale(r, c) * o)
    at = s["loose"]
    w[at] = (w[at].float() - ETA_REST * v[at]).to(w.dtype)
    return {"weights": w, "momentum": m}


def run(s):
    if not own:
        return _plain(s)
    call, plan = s["case"]["call"], s["plan"]
    if call == "norm_fwd":
        plan.artopk_layernorm_forward(s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], eps=LN_EPS)
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if call == "norm_bwd":
        plan.artopk_layernorm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"],
                                       s["dbeta"], accumulate=s["case"]["accumulate"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if call == "orth":
        plan.artopk_orthogonalize(s["x"], s["out"], steps=STEPS, eps=NORM_EPS)
        return {"out": s["out"]}
    plan.artopk_muon_step(s["weights"], s["momentum"], s["update"], eta=ETA, mu=MU, nesterov=s["case"]["nesterov"],
                          decay=DECAY, eta_rest=ETA_REST, steps=STEPS, eps=NORM_EPS)
    return {"weights": s["weights"], "momentum": s["momentum"]}


def work(case):
    size = 4 if case["type"] == "f32" else 2
    if case["call"] == "norm_fwd":
        r, c = case["rows"], case["cols"]
        return {"bytes": 2 * size * r * c + 8 * r + 8 * c, "flops": 8 * r * c}
    if case["call"] == "norm_bwd":
        r, c = case["rows"], case["cols"]
        return {"bytes": 3 * size * r * c + 8 * r + (20 if case["accumulate"] else 12) * c, "flops": 14 * r * c}
    mats, n = _matrices(case)
    inside = sum(r * c for _, r, c in mats)
    flops = sum(_flops(r, c) for _, r, c in mats)
    if case["call"] == "orth":
        return {"bytes": 2 * size * inside, "flops": flops}
    # update read, momentum and weights read and written
    return {"bytes": (12 + 2 * size) * n, "flops": flops + 4 * n}


# ---- the definitions in 64 bits ----------------------------------------------------------------
def _polar64(x, scale):
    """The same polynomial through the smaller Gram matrix alone: x_k = q_k x_0 (or x_0 q_k), with q_k and the
    Gram matrix of x_k both polynomials in the Gram matrix of x_0."""
    x = x.double()
    x = x / (torch.linalg.norm(x) + NORM_EPS)
    a, b, c = STEP
    wide = x.shape[0] <= x.shape[1]
    gram = torch.matmul(x, x.t().contiguous()) if wide else torch.matmul(x.t().contiguous(), x)
    one = torch.eye(gram.shape[0], dtype=torch.float64, device="cuda")
    q = one
    for _ in range(STEPS):
        p = a * one + torch.matmul(gram, b * one + c * gram)
        q = torch.matmul(p, q)
        gram = torch.matmul(torch.matmul(p, gram), p)
    return scale * (torch.matmul(q, x) if wide else torch.matmul(x, q))


def exact(case, seed):
    if case["call"].startswith("norm"):
        s = _norm_inputs(case, seed)
        x, gamma = s["x"].double(), s["gamma"].double()
        if case["call"] == "norm_fwd":
            var, mean = torch.var_mean(x, 1, correction=0)
            rstd = 1.0 / torch.sqrt(var + LN_EPS)
            y = torch.addcmul(s["beta"].double(), (x - mean[:, None]) * gamma, rstd[:, None].expand_as(x))
            return {"y": y, "mean": mean, "rstd": rstd}
        mean, rstd, dy = s["mean"].double(), s["rstd"].double(), s["dy"].double()
        hat = (x - mean[:, None]) * rstd[:, None]
        dgamma, dbeta = torch.mul(dy, hat).sum(0), dy.sum(0)
        one = torch.mv(dy, gamma) / case["cols"]
        two = torch.mv(dy * hat, gamma) / case["cols"]
        dx = (dy * gamma - one[:, None] - hat * two[:, None]) * rstd[:, None]
        if case["accumulate"]:
            dgamma, dbeta = dgamma + s["dgamma"].double(), dbeta + s["dbeta"].double()
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    s = _flat_inputs(case, seed)
    mats, n = _matrices(case)
    if case["call"] == "orth":
        out = torch.zeros(n, dtype=torch.float64, device="cuda")
        for at, r, c in mats:
            out[at:at + r * c] = _polar64(s["x"][at:at + r * c].view(r, c), _scale(r, c)).reshape(-1)
        return {"out": out}
    m = MU * s["momentum"].double() + s["update"].double()
    v = m.clone()
    if case["nesterov"]:
        v = MU * m + s["update"].double()
    w = s["weights"].double()
    new = w - ETA_REST * v
    for at, r, c in mats:
        o = _polar64(v[at:at + r * c].view(r, c), _scale(r, c)).reshape(-1)
        new[at:at + r * c] = (1.0 - ETA * DECAY) * w[at:at + r * c] - ETA * o
    return {"weights": new, "momentum": m}
