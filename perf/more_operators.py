"""The operators of the workers' models that hold matrix products, and what bounds a worker's gradient, call by call: what
stands between a hidden state and the rows of the gradient buffer that the optimizer's step reads.

Kinds of pass:

  gate_fwd  a gated feed-forward block up to its product: m = act(x Wg' + bg) * (x Wu' + bu); in training with the two
            projections kept for the backward pass, for answers without
  gate_bwd  the gradients of the two projections from those of m, and of the two biases for every worker
  proj_bwd  the gradients of what the two projections read, and of both weights for every worker
  lce       softmax cross-entropy of an output layer that is computed piece by piece and never kept, a worker's loss being
            the mean over its tokens, with the gradients of what it reads and of its weight for every worker
  clip      the norm of every worker's gradient, over many tensors, and the gradient cut to a largest one

`own` says which side runs: elementary torch operations in 32 bits, or the library's entry points.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
IGNORE = -100
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
KINDS = ["gate_fwd", "gate_bwd", "proj_bwd", "lce", "clip"]
ACTS = ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]


def _gated(name, kind, n, rows, cols, hidden, type, act="silu", pad=0, bias=True, keep=True):
    """n workers of `rows` rows each, `cols` columns projected to `hidden`.  pad: columns between the rows of the
    activations and of the weights.  keep: whether the projections are kept for a backward pass."""
    c = {"kind": kind, "n": n, "rows": rows, "cols": cols, "hidden": hidden, "type": type, "pad": pad}
    if kind != "proj_bwd":
        c.update(act=act, bias=bias)
    if kind == "gate_fwd":
        c["keep"] = keep
    return dict(c, name=name) if name else c


def _lce(name, n, rows, cols, vocab, type, pad=0, gradient=True):
    c = {"kind": "lce", "n": n, "rows": rows, "cols": cols, "vocab": vocab, "type": type, "pad": pad, "gradient": gradient}
    return dict(c, name=name) if name else c


def _clip(name, n, count, tensors, type, big=True, scale=1.0):
    """n workers' gradients of `count` entries in all, in `tensors` tensors.  big: whether the norms are above the largest
    one.  scale: the factor that takes a loss's scale back."""
    c = {"kind": "clip", "n": n, "count": count, "tensors": tensors, "type": type, "big": big, "scale": scale}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one sequence is answered: the weights are all there is to read
        _gated("gate_fwd_token", "gate_fwd", 1, 1, 768, 2048, "bf16", bias=False, keep=False),
        # eight workers with a sequence of 1024 tokens each, in training
        _gated("gate_fwd_gpt2s", "gate_fwd", 8, 1024, 768, 2048, "bf16"),
        # sizes nobody rounded, rows with a gap between them, half precision
        _gated("gate_fwd_odd", "gate_fwd", 5, 211, 777, 1111, "f16", act="gelu_tanh", pad=7),
        # the same model's gradients, projections and biases
        _gated("gate_bwd_gpt2s", "gate_bwd", 8, 1024, 768, 2048, "bf16"),
        # and of what the projections read and of their weights
        _gated("proj_bwd_gpt2s", "proj_bwd", 8, 1024, 768, 2048, "bf16"),
        # a small model's batch in full precision
        _gated("proj_bwd_small", "proj_bwd", 4, 512, 256, 768, "f32"),
        # a small model's next-token loss: few tokens, few of them to answer with
        _lce("lce_small", 4, 512, 256, 512, "f32"),
        # the loss of a text without its gradient, sizes nobody rounded
        _lce("lce_score", 3, 401, 777, 10007, "f16", pad=7, gradient=False),
        # the next-token loss of eight sequences of 1024 tokens with its gradients, the largest
        _lce("lce_gpt2s", 8, 1024, 768, 50257, "bf16"),
        # a small model's gradients, one row to a worker
        _clip("clip_tiny", 4, 65536, 1, "f32"),
        # one worker's gradients of many layers, as products in half precision left them, under a scaled loss
        _clip("clip_layers", 1, 1000003, 62, "f16", scale=2.0 ** -10),
        # sixteen workers' gradients of 11.2 million entries
        _clip("clip_r18", 16, 11181642, 1, "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(KINDS)
    n = rng.choice([1, 1, 2, 3, 4, 5, 8, 8, 16])
    type = rng.choice(["f32", "f16", "bf16", "bf16", "bf16"])
    pad = rng.choice([0, 0, 0, 1, 8, 24])
    if kind == "clip":
        count = _log_int(rng, 64, 150_000_000 // n)
        return _clip(None, n, count, min(count, rng.choice([1, 1, 2, 7, 62, 148])), type, big=rng.random() < 0.75,
                     scale=rng.choice([1.0, 1.0, 2.0 ** -10]))
    cols = _log_int(rng, 32, 4096)
    if kind == "lce":
        vocab = _log_int(rng, 32, 131072)
        gradient = rng.random() < 0.75
        most = min(16384, 300_000_000_000 // (cols * vocab), 400_000_000 // vocab)
        n = min(n, max(1, 300_000_000 // (cols * vocab)))
        return _lce(None, n, _log_int(rng, 1, max(2, most // n)), cols, vocab, type, pad, gradient)
    hidden = _log_int(rng, 32, 8192)
    most = min(16384, 100_000_000_000 // (cols * hidden), 130_000_000 // hidden)
    rows = _log_int(rng, 1, max(2, most // n))
    return _gated(None, kind, n, rows, cols, hidden, type, rng.choice(ACTS), pad, rng.random() < 0.5, rng.random() < 0.5)


# ---- inputs -----------------------------------------------------------------------------------------------

def _matrix(c, total, cols, type, g=None, scale=1.0):
    """A matrix whose rows are `pad` columns apart; filled with N(0, scale^2) from the generator, if one is given."""
    ld = cols + c["pad"]
    if g is None:
        return torch.empty((total, ld), dtype=TYPES[type], device=DEVICE)[:, :cols]
    return torch.randn((total, ld), generator=g, device=DEVICE).mul_(scale).to(TYPES[type])[:, :cols]


def _sizes(count, tensors):
    """The tensors' sizes: every third one is short (a bias beside its weight), the last takes what is left."""
    if tensors == 1:
        return [count]
    short = max(1, count // tensors // 64)
    sizes = [short if i % 3 else max(1, count // tensors) for i in range(tensors - 1)]
    return sizes + [count - sum(sizes)]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    kind, n, type = c["kind"], c["n"], c["type"]
    s = {"c": c}
    f32 = lambda *shape: torch.empty(shape, dtype=torch.float32, device=DEVICE)  # noqa: E731
    if kind == "clip":
        s["sizes"] = _sizes(c["count"], c["tensors"])
        s["tensors"] = []
        for k, size in enumerate(s["sizes"]):
            # layers differ in size, workers too
            std = 10.0 ** (-1.0 - (k * 7 % 5) / 4) * torch.linspace(0.5, 2.0, n, device=DEVICE)[:, None]
            s["tensors"].append((torch.randn((n, size), generator=g, device=DEVICE) * std).to(TYPES[type]))
        least = c["scale"] * 10.0 ** (-2.0) * math.sqrt(c["count"]) * 0.5
        s["max_norm"] = 0.1 * least if c["big"] else 1e4 * least
        # they go where the step reads them: side by side in the workers' rows
        s["rows"] = f32(n, c["count"])
        s["out"] = {"out": list(s["rows"].split(s["sizes"], 1)), "norms": f32(n), "factors": f32(n)}
        return s
    total, cols = n * c["rows"], c["cols"]
    small = 0.5 if type == "f16" else 1e-3    # half precision trains with a scaled loss
    if kind == "lce":
        vocab = c["vocab"]
        s["weight"] = _matrix(c, vocab, cols, type, g, 2.5 / math.sqrt(cols))
        t = torch.randint(0, vocab, (total,), generator=g, device=DEVICE)
        # a model that has learnt something: what it makes of a token looks a little like what comes next
        x = torch.randn((total, cols + c["pad"]), generator=g, device=DEVICE)
        x[:, :cols] += 0.64 * s["weight"][t].float()
        s["x"] = x.to(TYPES[type])[:, :cols]
        # a tenth of the tokens is padding that nothing is learnt from
        s["targets"] = torch.where(torch.rand(total, generator=g, device=DEVICE) < 0.1, IGNORE, t)
        s["grad_scale"] = 2.0 ** 10 if type == "f16" else 1.0
        s["out"] = {"mean_loss": f32(n), "losses": f32(total)}
        if c["gradient"]:
            s["out"].update(dx=_matrix(c, total, cols, type), dweight=f32(n, vocab, cols))
        return s
    hidden = c["hidden"]
    if kind == "gate_bwd":
        s["dm"] = _matrix(c, total, hidden, type, g, small)
        s["gate"] = _matrix(c, total, hidden, type, g)
        s["up"] = _matrix(c, total, hidden, type, g)
        s["out"] = {"dgate": _matrix(c, total, hidden, type), "dup": _matrix(c, total, hidden, type)}
        if c["bias"]:
            s["out"].update(dgate_bias=f32(n, hidden), dup_bias=f32(n, hidden))
        return s
    s["x"] = _matrix(c, total, cols, type, g)
    s["gate_weight"] = _matrix(c, hidden, cols, type, g, 1.0 / math.sqrt(cols))
    s["up_weight"] = _matrix(c, hidden, cols, type, g, 1.0 / math.sqrt(cols))
    if kind == "gate_fwd":
        bias = lambda: torch.randn(hidden, generator=g, device=DEVICE).mul_(0.1) if c["bias"] else None  # noqa: E731
        s["gate_bias"], s["up_bias"] = bias(), bias()
        s["out"] = {"m": _matrix(c, total, hidden, type)}
        if c["keep"]:
            s["out"].update(gate=_matrix(c, total, hidden, type), up=_matrix(c, total, hidden, type))
        return s
    s["dgate"] = _matrix(c, total, hidden, type, g, small)
    s["dup"] = _matrix(c, total, hidden, type, g, small)
    s["out"] = {"dx": _matrix(c, total, cols, type), "dgate_weight": f32(n, hidden, cols),
                "dup_weight": f32(n, hidden, cols)}
    return s


# ---- one pass ---------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2205_05632_amd import operators as ops
    c, kind, out = s["c"], s["c"]["kind"], s["out"]
    if kind == "gate_fwd":
        got = ops.compams_gated_forward(s["x"], s["gate_weight"], s["up_weight"], c["act"], gate_bias=s["gate_bias"],
                                        up_bias=s["up_bias"], keep=c["keep"], **out)
        return got if c["keep"] else got[:1]
    if kind == "gate_bwd":
        got = ops.compams_gated_backward(s["dm"], s["gate"], s["up"], c["n"], c["act"], bias=c["bias"], **out)
        return got if c["bias"] else got[:2]
    if kind == "proj_bwd":
        return ops.compams_projections_backward(s["dgate"], s["dup"], s["x"], s["gate_weight"], s["up_weight"], c["n"], **out)
    if kind == "lce":
        got = ops.compams_linear_cross_entropy(s["x"], s["weight"], s["targets"], c["n"], IGNORE, s["grad_scale"],
                                               gradient=c["gradient"], **out)
        return got if c["gradient"] else got[:2]
    _, norms, factors = ops.compams_clip_gradients(s["tensors"], s["max_norm"], c["n"], scale=c["scale"], **out)
    return s["rows"], norms, factors


# The plain form: 32 bits throughout (the norm's long sum in 64), each output rounded once.

def _act(a, act):
    """act(a) and its derivative."""
    if act == "relu":
        return torch.where(a > 0, a, torch.zeros_like(a)), (a > 0).to(a.dtype)
    if act == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
        return a * cdf, cdf + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        k = math.sqrt(2.0 / math.pi)
        t = torch.tanh(k * (a + 0.044715 * a * a * a))
        return 0.5 * a * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * a * a)
    q = 1.0 / (1.0 + torch.exp(-a))
    if act == "sigmoid":
        return q, q * (1.0 - q)
    return a * q, q * (1.0 + a * (1.0 - q))


def _by_worker(t, c):
    return t.reshape(c["n"], c["rows"], t.shape[1])


def _run_plain(s):
    c, kind = s["c"], s["c"]["kind"]
    type = TYPES[c["type"]]
    if kind == "gate_fwd":
        x = s["x"].float()
        a, b = x @ s["gate_weight"].float().t(), x @ s["up_weight"].float().t()
        if c["bias"]:
            a, b = a + s["gate_bias"], b + s["up_bias"]
        m = (_act(a, c["act"])[0] * b).to(type)
        return (m, a.to(type), b.to(type)) if c["keep"] else (m,)
    if kind == "gate_bwd":
        dm = s["dm"].float()
        value, slope = _act(s["gate"].float(), c["act"])
        da, db = dm * s["up"].float() * slope, dm * value
        if not c["bias"]:
            return da.to(type), db.to(type)
        return da.to(type), db.to(type), _by_worker(da, c).sum(1), _by_worker(db, c).sum(1)
    if kind == "proj_bwd":
        da, db, x = s["dgate"].float(), s["dup"].float(), s["x"].float()
        dx = da @ s["gate_weight"].float() + db @ s["up_weight"].float()
        xw = _by_worker(x, c)
        product = lambda d: torch.matmul(_by_worker(d, c).transpose(1, 2).contiguous(), xw)  # noqa: E731
        return dx.to(type), product(da), product(db)
    if kind == "clip":
        wide = [t.float() for t in s["tensors"]]
        norms = torch.sqrt(torch.stack([t.double().square().sum(1) for t in wide]).sum(0)) * c["scale"]
        factors = (c["scale"] * torch.clamp(s["max_norm"] / norms, max=1.0)).float()
        return torch.cat(wide, 1) * factors[:, None], norms.float(), factors
    x, w, t = s["x"].float(), s["weight"].float(), s["targets"]
    learnt = t != IGNORE
    count = learnt.reshape(c["n"], c["rows"]).sum(1)
    at = torch.where(learnt, t, torch.zeros_like(t))[:, None]
    logits = x @ w.t()
    top = logits.max(1, keepdim=True).values
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    losses = torch.where(learnt, (torch.log(total) + top - logits.gather(1, at))[:, 0], 0.0)
    mean = torch.where(count > 0, losses.reshape(c["n"], c["rows"]).sum(1) / count, 0.0)
    if not c["gradient"]:
        return mean, losses
    factor = torch.where(learnt, (s["grad_scale"] / count).repeat_interleave(c["rows"]), 0.0)[:, None]
    d = e / total
    d.scatter_add_(1, at, torch.full_like(total, -1.0))
    d = d * factor
    return mean, losses, (d @ w).to(type), torch.matmul(_by_worker(d, c).transpose(1, 2).contiguous(), _by_worker(x, c))


# ---- what a pass has to do ----------------------------------------------------------------------------------

def work(case):
    c = case
    kind, n, b = c["kind"], c["n"], SIZE[c["type"]]
    if kind == "clip":
        many = n * c["count"]
        return {"bytes": many * (b + 4) + 8 * n, "flops": 3 * many}
    total, cols = n * c["rows"], c["cols"]
    if kind == "lce":
        vocab = c["vocab"]
        read = (total + vocab) * cols * b + 12 * total + 4 * n
        if not c["gradient"]:
            return {"bytes": read, "flops": 2 * total * cols * vocab}
        return {"bytes": read + total * cols * b + 4 * n * vocab * cols, "flops": 6 * total * cols * vocab}
    hidden = c["hidden"]
    if kind == "gate_fwd":
        return {"bytes": (total + 2 * hidden) * cols * b + total * hidden * b * (3 if c["keep"] else 1)
                + (8 * hidden if c["bias"] else 0), "flops": 4 * total * cols * hidden}
    if kind == "gate_bwd":
        return {"bytes": 5 * total * hidden * b + (8 * n * hidden if c["bias"] else 0), "flops": 12 * total * hidden}
    return {"bytes": (2 * total + 2 * hidden) * cols * b + 2 * total * hidden * b + 8 * n * hidden * cols,
            "flops": 8 * total * cols * hidden}


# ---- the definition in 64 bits -------------------------------------------------------------------------------

def _linked64(a, act):
    """The activation of `a` with autograd's link to it."""
    if act == "relu":
        return torch.relu(a)
    if act == "gelu":
        return a * torch.special.ndtr(a)
    if act == "gelu_tanh":
        return a * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (a + 0.044715 * a.pow(3)))
    return torch.sigmoid(a) if act == "sigmoid" else a * torch.sigmoid(a)


def exact(case, seed):
    s = prepare(case, seed)
    s.pop("out")
    c, kind = s["c"], s["c"]["kind"]
    if kind == "clip":
        rows = torch.cat([t.double() for t in s["tensors"]], 1)
        norms = c["scale"] * torch.linalg.vector_norm(rows, dim=1)
        factors = c["scale"] * torch.minimum(s["max_norm"] / norms, torch.ones_like(norms))
        return rows.mul_(factors.unsqueeze(1)), norms, factors
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    split = lambda t: t.unflatten(0, (c["n"], c["rows"]))  # noqa: E731
    if kind == "gate_fwd":
        a = torch.nn.functional.linear(wide["x"], wide["gate_weight"], wide.get("gate_bias"))
        b = torch.nn.functional.linear(wide["x"], wide["up_weight"], wide.get("up_bias"))
        m = _linked64(a, c["act"]) * b
        return (m, a, b) if c["keep"] else (m,)
    if kind == "gate_bwd":
        a, b = wide["gate"].requires_grad_(True), wide["up"].requires_grad_(True)
        da, db = torch.autograd.grad(_linked64(a, c["act"]) * b, (a, b), wide["dm"])
        return (da, db, split(da).sum(1), split(db).sum(1)) if c["bias"] else (da, db)
    if kind == "proj_bwd":
        d = torch.cat([wide["dgate"], wide["dup"]], 1)
        dx = torch.mm(d, torch.cat([wide["gate_weight"], wide["up_weight"]], 0))
        dw = torch.stack([torch.mm(a.t(), b) for a, b in zip(split(d).unbind(0), split(wide["x"]).unbind(0))])
        return dx, dw[:, :c["hidden"]].contiguous(), dw[:, c["hidden"]:].contiguous()
    # a worker at a time
    means, losses, dxs, dws = [], [], [], []
    for x, t in zip(split(wide["x"]).unbind(0), s["targets"].unflatten(0, (c["n"], c["rows"])).unbind(0)):
        learnt = t.ne(IGNORE)
        at, count = t.clamp(min=0).unsqueeze(1), max(1, int(learnt.sum()))
        logp = torch.log_softmax(torch.mm(x, wide["weight"].t()), dim=1)
        losses.append(-logp.gather(1, at).squeeze(1) * learnt)
        means.append(losses[-1].sum() / count)
        if c["gradient"]:
            d = logp.exp_()
            d.scatter_(1, at, d.gather(1, at) - 1.0)
            d *= learnt.unsqueeze(1) * (s["grad_scale"] / count)
            dxs.append(torch.mm(d, wide["weight"]))
            dws.append(torch.mm(d.t(), x))
    mean, losses = torch.stack(means), torch.cat(losses)
    return (mean, losses, torch.cat(dxs), torch.stack(dws)) if c["gradient"] else (mean, losses)
