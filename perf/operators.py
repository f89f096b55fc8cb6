"""The operators of a language model's training step, as their users run them: the cases a change to their kernels is timed on.

Three operators ("op"), each for n workers that are batched buffers on one GPU, as everywhere in the library:

  norm    layer norm over the last axis; "train": forward and backward pass with the sums of the weight's and bias's
          gradients per worker; otherwise the forward pass alone.
  xent    the output layer and its softmax cross entropy, mean over a worker's labelled tokens; "train": the loss and
          the gradients of the hidden states and, per worker, of the weight; otherwise the loss alone.  Labels of -100
          mark tokens that take no part (their row of "lse" is 0).
  ortho   an update orthogonalised by five Newton-Schulz steps; "workers" > 0: the whole momentum update of weight
          matrices from that many workers' gradients; 0: the orthogonalisation by itself.

"type" is that of activations, weights and their gradients ("f32", "bf16", "f16"); norms' weights, losses, and momenta
and parameters of an update are always f32.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
STEPS, COEF, ORTHO_EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
BETA, LR, DECAY = 0.95, 0.02, 0.1
IGNORED = -100
WIDTHS = (32, 64, 96, 128, 192, 256, 320, 384, 512, 640, 768, 1024, 1280, 1536, 2048, 2560, 4096, 5120, 6144, 8192)


def _norm(name, n, t, dim, type, train):
    return {"name": name, "op": "norm", "n": n, "t": t, "dim": dim, "type": type, "train": train}


def _xent(name, n, t, dim, vocab, type, train):
    return {"name": name, "op": "xent", "n": n, "t": t, "dim": dim, "vocab": vocab, "type": type, "train": train}


def _ortho(name, workers, batch, rows, cols, type):
    return {"name": name, "op": "ortho", "workers": workers, "batch": batch, "rows": rows, "cols": cols, "type": type}


def listed():
    return [
        # a handful of tokens scored: launches and latencies
        _norm("norm-few", 4, 2, 512, "f32", False),
        # eight workers' sequences of 1024 tokens, the width of a language model of 124 million parameters
        _norm("norm-768", 8, 1024, 768, "bf16", True),
        # lengths and widths as they come, in full precision
        _norm("norm-ragged", 3, 1531, 1283, "f32", True),
        # long sequences of a wide model
        _norm("norm-wide", 4, 4096, 8192, "bf16", True),
        # a small model's head over a few tokens
        _xent("xent-few", 4, 5, 256, 4001, "f32", True),
        # scoring held-out text
        _xent("xent-eval", 1, 4096, 1024, 32000, "f16", False),
        # full precision, a sequence that lost its first token to the shift of the labels
        _xent("xent-f32", 4, 511, 768, 50257, "f32", True),
        # eight workers' batches in a language model of 124 million parameters
        _xent("xent-50257", 8, 1024, 768, 50257, "bf16", True),
        # a layer of a small network, fifty workers
        _ortho("muon-small-n50", 50, 1, 84, 120, "f32"),
        # twelve layers' square projections of a language model of 124 million parameters, eight workers
        _ortho("muon-768", 8, 12, 768, 768, "f32"),
        # tall matrices of odd sizes
        _ortho("ortho-ragged", 0, 3, 1531, 611, "f32"),
        # a large model's projection
        _ortho("ortho-large", 0, 1, 4096, 8192, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, size):
    """An odd size near `size`, or the next width below it that models are built with."""
    if rng.random() < 0.5:
        return size | 1
    return max((w for w in WIDTHS if w <= size), default=size)


def draw(rng):
    op = rng.choice(("norm", "xent", "ortho"))
    type = rng.choice(("f32", "bf16", "f16"))
    case = None
    if op == "norm":
        n, t, dim = rng.randint(1, 8), _log(rng, 1, 4096), _log(rng, 16, 8192)
        dim = _width(rng, dim)
        t = max(1, min(t, 4 * 4096 * 8192 // (n * dim * (2 if type == "f32" else 1))))
        case = _norm("", n, t, dim, type, rng.random() < 0.7)
    elif op == "xent":
        n, t, dim, vocab = rng.randint(1, 8), _log(rng, 1, 4096), _log(rng, 32, 2048), _log(rng, 500, 65536)
        dim = _width(rng, dim)
        t = max(1, min(t, 8 * 1024 * 768 * 50257 // (n * dim * vocab * (2 if type == "f32" else 1))))
        case = _xent("", n, t, dim, vocab, type, rng.random() < 0.7)
    else:
        batch, rows, cols = rng.randint(1, 12), _log(rng, 16, 4096), _log(rng, 16, 8192)
        rows, cols = _width(rng, rows), _width(rng, cols)
        workers = rng.choice((0, 0, rng.randint(1, 8)))
        limit = 2 * 4096 * 4096 * 8192 // (4 if workers or type == "f32" else 1)
        small, large = min(rows, cols), max(rows, cols)
        batch = max(1, min(batch, limit // (2 * small * small * large)))
        case = _ortho("", workers, batch, rows, cols, "f32" if workers else type)
        while work(case)["flops"] > work(_ortho("", 0, 1, 4096, 8192, "bf16"))["flops"] // 2:
            case["rows"], case["cols"] = max(16, case["rows"] * 7 // 8), max(16, case["cols"] * 7 // 8)
    del case["name"]
    return case


def _size(type):
    return 4 if type == "f32" else 2


def work(case):
    size = _size(case["type"])
    if case["op"] == "norm":
        elems = case["n"] * case["t"] * case["dim"]
        # forward: x in, y out; backward: x and dy in, dx out
        return {"bytes": elems * size * (5 if case["train"] else 2) + 8 * case["dim"] * (1 + case["n"]),
                "flops": elems * (18 if case["train"] else 7)}
    if case["op"] == "xent":
        rows, dim, vocab, n = case["n"] * case["t"], case["dim"], case["vocab"], case["n"]
        moved = (rows * dim + vocab * dim) * size + rows * 12
        if case["train"]:
            moved += (rows * dim + n * vocab * dim) * size
        return {"bytes": moved, "flops": 2 * rows * dim * vocab * (3 if case["train"] else 1)}
    elems, small, large = case["batch"] * case["rows"] * case["cols"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # a step's products: the Gram matrix and its square, of which half is enough by symmetry, and the product with X
    flops = STEPS * case["batch"] * (small * small * large + small ** 3 + 2 * small * small * large)
    moved = elems * size * (2 if not case["workers"] else case["workers"] + 4)
    return {"bytes": moved, "flops": flops}


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _inputs(case, seed):
    """The inputs of a case, from the seed alone."""
    gen, kind = _generator(seed), TYPES[case["type"]]
    if case["op"] == "norm":
        n, t, dim = case["n"], case["t"], case["dim"]
        # hidden states: a common offset and scale per feature, some features far larger than the others
        scale = torch.exp(0.5 * _randn(gen, dim))
        scale[:: max(1, dim // 7)] *= 8
        x = (_randn(gen, n, t, dim) * scale + 0.3 * _randn(gen, dim)).to(kind)
        s = {"x": x, "weight": 1 + 0.2 * _randn(gen, dim), "bias": 0.1 * _randn(gen, dim)}
        if case["train"]:
            s["dy"] = (_randn(gen, n, t, dim) * torch.exp(_randn(gen, n, t, 1)) / t).to(kind)
        return s
    if case["op"] == "xent":
        n, t, dim, vocab = case["n"], case["t"], case["dim"], case["vocab"]
        w = (_randn(gen, vocab, dim) * 0.05).to(kind)
        labels = (torch.rand((n, t), generator=gen, device="cuda") ** 3 * vocab).long().clamp_(max=vocab - 1)
        # hidden states as after a norm, leaning to their labels: a model that has learnt something
        h = (_randn(gen, n, t, dim) + 2.0 * w.float()[labels] / (0.05 * math.sqrt(dim)) * torch.rand((n, t, 1), generator=gen, device="cuda") * math.sqrt(dim) / 8)
        labels[torch.rand((n, t), generator=gen, device="cuda") < 0.06] = IGNORED
        return {"h": h.to(kind), "w": w, "labels": labels}
    batch, rows, cols, workers = case["batch"], case["rows"], case["cols"], case["workers"]

    def update(count):
        # a few strong directions over a slowly falling spectrum, as gradients of weight matrices have
        rank = min(rows, cols, 16)
        strong = (_randn(gen, count, rows, rank) / torch.arange(1, rank + 1, device="cuda")) @ _randn(gen, count, rank, cols)
        return (strong * 0.2 + _randn(gen, count, rows, cols)) * 1e-3

    if not workers:
        return {"g": update(batch).to(kind)}
    common = update(batch)
    g = torch.empty((workers, batch, rows, cols), device="cuda")
    for i in range(workers):
        g[i] = common + 1e-3 * _randn(gen, batch, rows, cols)
    return {"g": g, "m": common + 3e-4 * _randn(gen, batch, rows, cols), "x": 0.02 * _randn(gen, batch, rows, cols)}


def _scale(case):
    return math.sqrt(max(1.0, case["rows"] / case["cols"]))


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if not own:
        return s
    from paper_2210_07454_amd import sams
    kind = TYPES[case["type"]]
    if case["op"] == "norm":
        n, t, dim = case["n"], case["t"], case["dim"]
        s["plan"] = sams.LayerNorm(n, t, dim, kind)
        s["y"] = torch.empty_like(s["x"])
        s["mean"], s["rstd"] = torch.empty((2, n, t), device="cuda")
        if case["train"]:
            s["dx"] = torch.empty_like(s["x"])
            s["dweight"], s["dbias"] = torch.empty((2, n, dim), device="cuda")
    elif case["op"] == "xent":
        n, t, dim, vocab = case["n"], case["t"], case["dim"], case["vocab"]
        s["plan"] = sams.LinearCrossEntropy(n, t, dim, vocab, kind, train=case["train"])
        s["loss"], s["lse"] = torch.empty((n,), device="cuda"), torch.empty((n, t), device="cuda")
        if case["train"]:
            s["dh"], s["dw"] = torch.empty_like(s["h"]), torch.empty((n, vocab, dim), device="cuda", dtype=kind)
    else:
        s["plan"] = sams.Orthogonalizer(case["batch"], case["rows"], case["cols"], kind)
        if case["workers"]:
            s["m_out"], s["x_out"] = torch.empty_like(s["m"]), torch.empty_like(s["x"])
        else:
            s["out"] = torch.empty_like(s["g"])
    return s


def run(state):
    case = state["case"]
    if own:
        return {"norm": _own_norm, "xent": _own_xent, "ortho": _own_ortho}[case["op"]](case, state)
    return {"norm": _plain_norm, "xent": _plain_xent, "ortho": _plain_ortho}[case["op"]](case, state)


# ---- the library's operators ----
def _own_norm(case, s):
    s["plan"].layer_norm_forward(s["x"], s["weight"], s["bias"], s["y"], s["mean"], s["rstd"], EPS)
    if not case["train"]:
        return [s["y"]]
    s["plan"].layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"], s["dbias"])
    return [s["y"], s["dx"], s["dweight"], s["dbias"]]


def _own_xent(case, s):
    s["plan"].linear_xent_forward(s["h"], s["w"], s["labels"], s["loss"], s["lse"])
    if not case["train"]:
        return [s["loss"], s["lse"]]
    s["plan"].linear_xent_backward(s["h"], s["w"], s["labels"], s["lse"], None, s["dh"], s["dw"])
    return [s["loss"], s["lse"], s["dh"], s["dw"]]


def _own_ortho(case, s):
    if not case["workers"]:
        s["plan"].orthogonalize(s["g"], s["out"], steps=STEPS, coef=COEF, eps=ORTHO_EPS)
        return [s["out"]]
    s["plan"].muon_update(s["g"], s["m"], s["x"], s["m_out"], s["x_out"], beta=BETA, nesterov=True, lr=LR, scale=_scale(case),
                          weight_decay=DECAY, steps=STEPS, coef=COEF, eps=ORTHO_EPS)
    return [s["m_out"], s["x_out"]]


# ---- the plain form: elementary operations in 32 bits, rounded once at the end ----
def _plain_norm(case, s):
    kind = s["x"].dtype
    x = s["x"].float()
    centred = x - x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt((centred * centred).mean(-1, keepdim=True) + EPS)
    xhat = centred * rstd
    y = (xhat * s["weight"] + s["bias"]).to(kind)
    if not case["train"]:
        return [y]
    dy = s["dy"].float()
    scaled = dy * s["weight"]
    dx = rstd * (scaled - scaled.mean(-1, keepdim=True) - xhat * (scaled * xhat).mean(-1, keepdim=True))
    return [y, dx.to(kind), (dy * xhat).sum(1), dy.sum(1)]


def _plain_xent(case, s):
    kind, (n, t, dim) = s["h"].dtype, s["h"].shape
    h, w, labels = s["h"].float().reshape(n * t, dim), s["w"].float(), s["labels"].reshape(-1)
    used = labels >= 0
    safe = torch.where(used, labels, 0)
    z = h @ w.t()
    top = z.amax(1, keepdim=True)
    shifted = torch.exp(z - top)
    total = shifted.sum(1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    lse = torch.where(used, lse, 0.0)
    per_token = torch.where(used, lse - z.gather(1, safe[:, None]).squeeze(1), 0.0).reshape(n, t)
    count = used.reshape(n, t).sum(1).clamp(min=1).float()
    loss = per_token.sum(1) / count
    if not case["train"]:
        return [loss, lse.reshape(n, t)]
    dz = shifted / total
    rows = torch.arange(n * t, device=h.device)
    dz[rows, safe] -= 1
    dz *= (used.reshape(n, t).float() / count[:, None]).reshape(-1, 1)
    dh = (dz @ w).reshape(n, t, dim).to(kind)
    dw = torch.empty((n, w.shape[0], dim), dtype=kind, device=h.device)
    for i in range(n):
        dw[i] = (dz[i * t:(i + 1) * t].t() @ h[i * t:(i + 1) * t]).to(kind)
    return [loss, lse.reshape(n, t), dh, dw]


def _plain_orthogonal(g):
    x = g.transpose(1, 2).contiguous() if g.shape[1] > g.shape[2] else g
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + ORTHO_EPS)
    a, b, c = COEF
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(1, 2).contiguous() if g.shape[1] > g.shape[2] else x


def _plain_ortho(case, s):
    if not case["workers"]:
        return [_plain_orthogonal(s["g"].float()).to(s["g"].dtype)]
    mean = s["g"].sum(0) / case["workers"]
    m = BETA * s["m"] + (1 - BETA) * mean
    update = _plain_orthogonal(BETA * m + (1 - BETA) * mean)
    return [m, (1 - LR * DECAY) * s["x"] - (LR * _scale(case)) * update]


# ---- the definitions in 64 bits ----
def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "xent": _exact_xent, "ortho": _exact_ortho}[case["op"]](case, s)


def _exact_norm(case, s):
    x, w, b = s["x"].double(), s["weight"].double(), s["bias"].double()
    var, mean = torch.var_mean(x, dim=-1, unbiased=False, keepdim=True)
    deviation = torch.sqrt(var + EPS)
    z = (x - mean) / deviation
    out = [z * w + b]
    if case["train"]:
        dy, dim = s["dy"].double(), case["dim"]
        dz = dy * w
        # the Jacobian of z is (I - (1 1' + z z') / dim) / deviation
        out.append((dz - (dz.sum(-1, keepdim=True) + z * (dz * z).sum(-1, keepdim=True)) / dim) / deviation)
        out.append(torch.einsum("ntd,ntd->nd", dy, z))
        out.append(dy.sum(1))
    return out


def _exact_xent(case, s):
    n, t, dim = s["h"].shape
    vocab, w = case["vocab"], s["w"].double()
    loss = torch.zeros(n, dtype=torch.float64, device="cuda")
    lse = torch.zeros((n, t), dtype=torch.float64, device="cuda")
    dh = torch.empty((n, t, dim), dtype=torch.float64, device="cuda") if case["train"] else None
    dw = torch.empty((n, vocab, dim), dtype=torch.float64, device="cuda") if case["train"] else None
    for i in range(n):
        h, labels = s["h"][i].double(), s["labels"][i]
        used = (labels != IGNORED).nonzero().squeeze(1)
        count = max(1, used.numel())
        logp = torch.log_softmax(h @ w.t(), dim=1)
        lse[i, used] = (h @ w[0] - logp[:, 0])[used]
        loss[i] = -logp[used, labels[used]].sum() / count
        if case["train"]:
            p = torch.zeros((t, vocab), dtype=torch.float64, device="cuda")
            p[used] = logp[used].exp()
            p[used, labels[used]] -= 1
            dh[i] = p @ w / count
            dw[i] = p.t() @ h / count
    return [loss, lse] + ([dh, dw] if case["train"] else [])


def _exact_orthogonal(g):
    out = torch.empty_like(g)
    for i in range(g.shape[0]):
        x = g[i] / (torch.linalg.matrix_norm(g[i]) + ORTHO_EPS)
        small = min(x.shape)
        one = torch.eye(small, dtype=torch.float64, device=g.device)
        for _ in range(STEPS):
            # on the shorter side; p(s) = s (a + s^2 (b + c s^2)) on every singular value s
            q = x @ x.t() if x.shape[0] == small else x.t() @ x
            poly = COEF[0] * one + q @ (COEF[1] * one + COEF[2] * q)
            x = poly @ x if x.shape[0] == small else x @ poly
        out[i] = x
    return out


def _exact_ortho(case, s):
    if not case["workers"]:
        return [_exact_orthogonal(s["g"].double())]
    mean = s["g"].double().mean(0)
    m = s["m"].double().lerp(mean, 1 - BETA)
    update = _exact_orthogonal(m.lerp(mean, 1 - BETA))
    return [m, s["x"].double() * (1 - LR * DECAY) - LR * _scale(case) * update]
