"""The operators of the workers' models whose speed is followed: what the forward and backward pass that fills the rows
of the gradient buffer asks of this library around its matrix products, call by call.

Kinds of pass:

  ln_fwd    layer norm of every row, with the statistics that the backward pass takes
  ln_bwd    its gradient: of the input, and of the two weights for every worker (a worker's rows follow each other)
  drop      dropout from a counter-based generator, alone or added to the residual stream (its own backward pass too)
  dan_fwd   the join between two branches of a transformer block: bias, dropout, residual add and layer norm
  dan_bwd   its gradient: of the branch, of the residual stream, of the norm's weights and of the bias for every worker
  ce        softmax cross-entropy with its gradient, a worker's loss being the mean over its tokens

`own` says which side runs: elementary torch operations in 32 bits, or the library's entry points.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-5
IGNORE = -100
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
KINDS = ["ln_fwd", "ln_bwd", "drop", "dan_fwd", "dan_bwd", "ce"]


def _case(name, kind, n, rows, cols, branch, stream, pad=0, p=0.1, residual=True, masked="none"):
    """n workers of `rows` rows each, `cols` columns.  branch: the type of what matrix products read and write (x, y,
    dy, dx, logits); stream: the type of the residual stream (for drop: of the output).  pad: columns between the rows.
    residual: whether dropout is added to one.  masked: what stands in a tenth of the vocabulary ("none": nothing
    special, "inf": minus infinity, "lowest": the type's lowest value)."""
    c = {"kind": kind, "n": n, "rows": rows, "cols": cols, "branch": branch, "stream": stream, "pad": pad}
    if kind in ("drop", "dan_fwd", "dan_bwd"):
        c["p"] = p
    if kind == "drop":
        c["residual"] = residual
    if kind == "ce":
        c["masked"] = masked
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of each of sixteen sequences: a launch and next to no bytes
        _case("ln_fwd_few", "ln_fwd", 1, 16, 768, "f32", "f32"),
        # eight workers with eight sequences of 1024 tokens each, a stream in 32 bits normed for a product in bfloat16
        _case("ln_fwd_gpt2s", "ln_fwd", 8, 8192, 768, "bf16", "f32"),
        # the same model with a sequence to a worker: the gradient
        _case("ln_bwd_gpt2s", "ln_bwd", 8, 1024, 768, "bf16", "f32"),
        # sizes nobody rounded, rows with a gap between them, half precision throughout
        _case("ln_bwd_odd", "ln_bwd", 5, 211, 1111, "f16", "f16", pad=7),
        # the embedding's dropout of eight sequences
        _case("drop_embed", "drop", 8, 1024, 768, "f32", "f32", residual=False),
        # the dropout of four sequences' attention weights, twelve heads of 1024 x 1024
        _case("drop_weights", "drop", 4, 12288, 1024, "bf16", "bf16", residual=False),
        # four tokens to a worker: a short answer, a probe
        _case("dan_fwd_few", "dan_fwd", 8, 4, 768, "bf16", "f32"),
        # the join of a whole batch, forward and backward
        _case("dan_fwd_gpt2s", "dan_fwd", 8, 8192, 768, "bf16", "f32"),
        _case("dan_bwd_gpt2s", "dan_bwd", 8, 8192, 768, "bf16", "f32"),
        # an ordinary small batch of a width nobody rounded
        _case("dan_bwd_odd", "dan_bwd", 3, 401, 1601, "bf16", "bf16"),
        # a batch of 32 pictures to a worker over 1000 classes
        _case("ce_classes", "ce", 8, 32, 1000, "f32", "f32"),
        # the next-token loss of eight sequences of 1024 tokens, the largest: rows of an odd vocabulary one after another
        _case("ce_gpt2s", "ce", 8, 1024, 50257, "bf16", "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(KINDS)
    n = rng.choice([1, 1, 2, 3, 4, 5, 8, 8, 16])
    branch, stream = rng.choice([("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f32"),
                                 ("bf16", "f32")])
    if kind == "ce":
        cols, stream, most = _log_int(rng, 32, 131072), branch, 400_000_000
    else:
        cols, most = _log_int(rng, 32, 12288), 50_000_000
    rows = _log_int(rng, 1, max(2, min(16384, most // (n * cols) // (2 if branch == "f32" else 1))))
    pad = rng.choice([0, 0, 0, 1, 8, 24])
    return _case(None, kind, n, rows, cols, branch, stream, pad=pad, p=rng.choice([0.0, 0.05, 0.1, 0.1, 0.2, 0.5]),
                 residual=rng.random() < 0.5, masked=rng.choice(["none", "none", "inf", "lowest"]))


# ---- inputs -----------------------------------------------------------------------------------------------

def _rows(c, kind, g=None, scale=1.0):
    """A tensor of the case's rows, `pad` columns apart; filled with N(0, scale^2) from the generator, if one is given."""
    total, cols, ld = c["n"] * c["rows"], c["cols"], c["cols"] + c["pad"]
    if g is None:
        return torch.empty((total, ld), dtype=TYPES[kind], device=DEVICE)[:, :cols]
    t = torch.randn((total, ld), generator=g, device=DEVICE)
    return t.mul_(scale).to(TYPES[kind])[:, :cols]


def _stream(c, g):
    """The residual stream: N(0,1) with a few channels that are much larger, as trained transformers have them."""
    t = torch.randn((c["n"] * c["rows"], c["cols"] + c["pad"]), generator=g, device=DEVICE)
    t[:, :: 97] *= 6.0
    return t.to(TYPES[c["stream"]])[:, : c["cols"]]


def _stats(h):
    f = h.float()
    mean = f.mean(1)
    return mean, torch.rsqrt((f - mean[:, None]).square().mean(1) + EPS)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    kind, total, cols, n = c["kind"], c["n"] * c["rows"], c["cols"], c["n"]
    s = {"c": c, "seed": (int(seed) * 0x9E3779B97F4A7C15 + 12345) % (1 << 64), "offset": 3 + (int(seed) << 20)}
    vector = lambda count: torch.empty(count, dtype=torch.float32, device=DEVICE)  # noqa: E731
    weight = lambda: torch.empty((n, cols), dtype=torch.float32, device=DEVICE)    # noqa: E731
    if kind == "ce":
        x = torch.randn((total, cols + c["pad"]), generator=g, device=DEVICE).mul_(2.5)
        t = torch.randint(0, cols, (total,), generator=g, device=DEVICE)
        if c["masked"] != "none":     # every tenth entry is none that this model may answer with
            lowest = torch.finfo(TYPES[c["branch"]]).min
            x[:, 3:cols:10] = -math.inf if c["masked"] == "inf" else lowest
            t = torch.where(t % 10 == 3, t - 1, t)
        x[torch.arange(total, device=DEVICE), t] += 4.0
        s["logits"] = x.to(TYPES[c["branch"]])[:, :cols]
        # a tenth of the tokens is padding that nothing is learnt from
        s["targets"] = torch.where(torch.rand(total, generator=g, device=DEVICE) < 0.1, IGNORE, t)
        # half precision trains with a scaled loss
        s["grad_scale"] = float(2 ** 15) if c["branch"] == "f16" else 1.0
        s["out"] = {"mean_loss": vector(n), "losses": vector(total), "dlogits": _rows(c, c["branch"])}
        return s
    if kind == "drop":
        s["x"] = _rows(c, c["branch"], g)
        s["residual"] = _stream(c, g) if c["residual"] else None
        s["out"] = {"y": _rows(c, c["stream"])}
        return s
    s["gamma"] = torch.randn(cols, generator=g, device=DEVICE).mul_(0.2).add_(1.0)
    s["beta"] = torch.randn(cols, generator=g, device=DEVICE).mul_(0.1)
    if kind == "ln_fwd":
        s["x"] = _stream(c, g)
        s["out"] = {"y": _rows(c, c["branch"]), "mean": vector(total), "rstd": vector(total)}
    elif kind == "dan_fwd":
        s["x"], s["residual"] = _rows(c, c["branch"], g), _stream(c, g)
        s["bias"] = torch.randn(cols, generator=g, device=DEVICE).mul_(0.1)
        s["out"] = {"h": _rows(c, c["stream"]), "y": _rows(c, c["branch"]), "mean": vector(total), "rstd": vector(total)}
    else:
        s["h"] = _stream(c, g)
        s["mean"], s["rstd"] = _stats(s["h"])
        size = 0.5 if c["branch"] == "f16" else 1e-3    # half precision trains with a scaled loss
        s["dy"] = _rows(c, c["branch"], g, size)
        s["out"] = {"dx": _rows(c, c["stream"] if kind == "ln_bwd" else c["branch"]), "dgamma": weight(),
                    "dbeta": weight()}
        if kind == "dan_bwd":
            s["dh"] = _rows(c, c["stream"], g, size)
            s["out"].update(dresidual=_rows(c, c["stream"]), dbias=weight())
    return s


# ---- one pass ---------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2205_05632_amd import operators as ops
    c, kind, out = s["c"], s["c"]["kind"], s["out"]
    if kind == "ln_fwd":
        return ops.compams_layer_norm_forward(s["x"], s["gamma"], s["beta"], EPS, **out)
    if kind == "ln_bwd":
        return ops.compams_layer_norm_backward(s["dy"], s["h"], s["mean"], s["rstd"], s["gamma"], c["n"], **out)
    if kind == "drop":
        return ops.compams_dropout(s["x"], c["p"], s["seed"], s["offset"], residual=s["residual"], **out)
    if kind == "dan_fwd":
        return ops.compams_dropout_add_norm_forward(s["x"], s["residual"], s["gamma"], s["beta"], c["p"], s["seed"],
                                                    s["offset"], EPS, bias=s["bias"], **out)
    if kind == "dan_bwd":
        return ops.compams_dropout_add_norm_backward(s["dy"], s["dh"], s["h"], s["mean"], s["rstd"], s["gamma"], c["p"],
                                                     s["seed"], s["offset"], c["n"], **out)
    return ops.compams_cross_entropy(s["logits"], s["targets"], c["n"], IGNORE, s["grad_scale"], **out)


# The plain form: 32 bits throughout, each output rounded once.

LOW = 0xFFFFFFFF


def _philox(counter, key):
    """Philox-4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011) on
    words held in 64-bit integers."""
    a, b, c, d = counter
    k0, k1 = key
    for _ in range(10):
        u, v = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = (((v >> 32) & LOW) ^ b ^ k0, v & LOW, ((u >> 32) & LOW) ^ d ^ k1, u & LOW)
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    return a, b, c, d


def _threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _kept(c, seed, offset):
    """Which entries are kept: column j of row r takes the (j mod 8)-th 16 bits of the words that the generator gives for
    the counter (j div 8, r, offset) and the key `seed`."""
    total, cols = c["n"] * c["rows"], c["cols"]
    blocks = (cols + 7) // 8
    one = torch.zeros((total, blocks), dtype=torch.int64, device=DEVICE)
    w = _philox((one + torch.arange(blocks, device=DEVICE), one + torch.arange(total, device=DEVICE)[:, None],
                 one + (offset & LOW), one + (offset >> 32)), (seed & LOW, seed >> 32))
    halves = torch.stack([w[0] & 0xFFFF, w[0] >> 16, w[1] & 0xFFFF, w[1] >> 16, w[2] & 0xFFFF, w[2] >> 16,
                          w[3] & 0xFFFF, w[3] >> 16], 2)
    return halves.reshape(total, 8 * blocks)[:, :cols] >= _threshold(c["p"])


def _dropped(v, c, seed, offset):
    scale = 65536.0 / (65536 - _threshold(c["p"]))
    return torch.where(_kept(c, seed, offset), v * scale, torch.zeros_like(v))


def _norm(h, gamma, beta):
    mean = h.sum(1) / h.shape[1]
    d = h - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).sum(1) / h.shape[1] + EPS)
    return d * rstd[:, None] * gamma + beta, mean, rstd


def _norm_backward(s):
    c = s["c"]
    dy, cols = s["dy"].float(), c["cols"]
    xhat = (s["h"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    a = dy * s["gamma"]
    dx = (a - (a.sum(1) / cols)[:, None] - xhat * ((a * xhat).sum(1) / cols)[:, None]) * s["rstd"][:, None]
    by_worker = lambda t: t.reshape(c["n"], c["rows"], cols).sum(1)  # noqa: E731
    return dx, by_worker(dy * xhat), by_worker(dy), by_worker


def _run_plain(s):
    c, kind = s["c"], s["c"]["kind"]
    branch, stream = TYPES[c["branch"]], TYPES[c["stream"]]
    if kind == "ln_fwd":
        y, mean, rstd = _norm(s["x"].float(), s["gamma"], s["beta"])
        return y.to(branch), mean, rstd
    if kind == "ln_bwd":
        dx, dgamma, dbeta, _ = _norm_backward(s)
        return dx.to(stream), dgamma, dbeta
    if kind == "drop":
        y = _dropped(s["x"].float(), c, s["seed"], s["offset"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return y.to(stream)
    if kind == "dan_fwd":
        h = s["residual"].float() + _dropped(s["x"].float() + s["bias"], c, s["seed"], s["offset"])
        y, mean, rstd = _norm(h, s["gamma"], s["beta"])
        return h.to(stream), y.to(branch), mean, rstd
    if kind == "dan_bwd":
        dres, dgamma, dbeta, by_worker = _norm_backward(s)
        dres = dres + s["dh"].float()
        dx = _dropped(dres, c, s["seed"], s["offset"])
        return dx.to(branch), dres.to(stream), dgamma, dbeta, by_worker(dx)
    x, t = s["logits"].float(), s["targets"]
    learnt = t != IGNORE
    count = learnt.reshape(c["n"], c["rows"]).sum(1)
    at = torch.where(learnt, t, torch.zeros_like(t))[:, None]
    top = x.max(1, keepdim=True).values
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    losses = torch.where(learnt, (torch.log(total) + top - x.gather(1, at))[:, 0], 0.0)
    mean = torch.where(count > 0, losses.reshape(c["n"], c["rows"]).sum(1) / count, 0.0)
    factor = torch.where(learnt, (s["grad_scale"] / count).repeat_interleave(c["rows"]), 0.0)[:, None]
    d = e / total
    d.scatter_add_(1, at, torch.full_like(total, -1.0))
    return mean, losses, (d * factor).to(branch)


# ---- what a pass has to do ----------------------------------------------------------------------------------

def work(case):
    c = case
    total, cols, n = c["n"] * c["rows"], c["cols"], c["n"]
    many, b, h = total * cols, SIZE[c["branch"]], SIZE[c["stream"]]
    kind = c["kind"]
    if kind == "ln_fwd":
        return {"bytes": many * (h + b) + 8 * cols + 8 * total, "flops": 8 * many}
    if kind == "ln_bwd":
        return {"bytes": many * (2 * h + b) + 4 * cols + 8 * total + 8 * n * cols, "flops": 15 * many}
    if kind == "drop":
        return {"bytes": many * (b + h + (h if c["residual"] else 0)), "flops": 2 * many}
    if kind == "dan_fwd":
        return {"bytes": many * (2 * b + 2 * h) + 12 * cols + 8 * total, "flops": 12 * many}
    if kind == "dan_bwd":
        return {"bytes": many * (2 * b + 3 * h) + 4 * cols + 8 * total + 12 * n * cols, "flops": 19 * many}
    return {"bytes": many * 2 * b + 12 * total + 4 * n, "flops": 6 * many}


# ---- the definition in 64 bits -------------------------------------------------------------------------------

def _mask64(c, seed, offset):
    """The kept entries, on the host: the generator's rounds in unsigned 64-bit numbers."""
    total, cols = c["n"] * c["rows"], c["cols"]
    blocks = -(-cols // 8)
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    x = np.empty((4, total, blocks), dtype=np.uint64)
    x[0], x[1] = np.arange(blocks, dtype=np.uint64)[None], np.arange(total, dtype=np.uint64)[:, None]
    x[2], x[3] = np.uint64(offset % 2 ** 32), np.uint64(offset // 2 ** 32)
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for turn in range(10):
        first, second = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        keys = [np.uint64((key[0] + turn * 0x9E3779B9) % 2 ** 32), np.uint64((key[1] + turn * 0xBB67AE85) % 2 ** 32)]
        x[0], x[2] = (second >> half) ^ x[1] ^ keys[0], (first >> half) ^ x[3] ^ keys[1]
        x[1], x[3] = second & low, first & low
    parts = np.ascontiguousarray(x.astype("<u4").transpose(1, 2, 0)).view("<u2").reshape(total, 8 * blocks)
    return torch.from_numpy(parts[:, :cols].astype(np.int32) >= math.floor(c["p"] * 65536 + 0.5)).to(DEVICE)


def _drop64(v, c, s):
    left = 65536 - math.floor(c["p"] * 65536 + 0.5)
    return (v * (65536 / left)).masked_fill_(~_mask64(c, s["seed"], s["offset"]), 0.0)


def exact(case, seed):
    s = prepare(case, seed)
    s.pop("out")
    c, kind = s["c"], s["c"]["kind"]
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if kind == "drop":
        y = _drop64(wide["x"], c, s)
        return y + wide["residual"] if c["residual"] else y
    if kind in ("ln_fwd", "dan_fwd"):
        h = wide["x"] if kind == "ln_fwd" else _drop64(wide["x"] + wide["bias"], c, s) + wide["residual"]
        var, mean = torch.var_mean(h, dim=1, correction=0)
        rstd = (var + EPS).pow(-0.5)
        y = torch.addcmul(wide["beta"], (h - mean.unsqueeze(1)) * rstd.unsqueeze(1), wide["gamma"])
        return (y, mean, rstd) if kind == "ln_fwd" else (h, y, mean, rstd)
    if kind in ("ln_bwd", "dan_bwd"):
        # y = gamma * z + beta with z = (h - mean) * rstd: dh = rstd * (I - 11'/C - zz'/C) (gamma * dy), for the
        # statistics as they were saved
        dy, r = wide["dy"], wide["rstd"].unsqueeze(1)
        z = (wide["h"] - wide["mean"].unsqueeze(1)) * r
        u = dy * wide["gamma"]
        d = r * (u - u.mean(1, keepdim=True) - z * (z * u).mean(1, keepdim=True))
        total = lambda t: t.unflatten(0, (c["n"], c["rows"])).sum(dim=1)  # noqa: E731
        if kind == "ln_bwd":
            return d, total(dy * z), total(dy)
        d += wide["dh"]
        dx = _drop64(d, c, s)
        return dx, d, total(dy * z), total(dy), total(dx)
    logp = torch.log_softmax(wide["logits"], dim=1)
    learnt = s["targets"].ne(IGNORE)
    at = s["targets"].clamp(min=0).unsqueeze(1)
    losses = -logp.gather(1, at).squeeze(1) * learnt
    share = learnt.unflatten(0, (c["n"], c["rows"])).sum(1).double()
    d = logp.exp_()
    d.scatter_(1, at, d.gather(1, at) - 1.0)
    d *= (learnt / share.clamp(min=1.0).repeat_interleave(c["rows"]) * s["grad_scale"]).unsqueeze(1)
    return losses.unflatten(0, (c["n"], c["rows"])).sum(1) / share.clamp(min=1.0), losses, d
