"""The operators that hold matrix products, and the bound of a gradient, from their formulas in 64 bits on the host, with the
error that each entry may have.

Bounds.  U = 2^-24.  A product's sum of K terms may be added up in any order, with an error of 2 U (a truncation) of what has
been added up at every addition and U at every product: at most (2 K + 4) U times the sum of the terms' magnitudes.  exp(z)
is off by (|z| + 3) U of itself (the product with log2 e, the processor's 2^x to a unit), 1 / x by 2 U, erfc by 40 U and by
2 z^2 times its argument's U (its relative slope).  Outputs are then rounded once (half a step, `unit(T)`).
"""
import math

import torch

from operator_reference import LEAST, U, UNIT, close, rounding  # noqa: F401

# A sigmoid below e^-88 = 2^-127 may be 0, and what follows from it with it: up to |a| (1 + inner) <= 20 * 30 times as much.
TINY = 2.0 ** -117


def sums(a, b, terms):
    """The error of a @ b where `terms` terms are added up."""
    return (2 * terms + 4) * U * (a.abs() @ b.abs())


def activation(a, name):
    """act(a), its derivative, and the errors of both for this a."""
    if name == "relu":
        one = (a > 0).double()
        return torch.where(torch.isnan(a), a, a * one), torch.where(torch.isnan(a), a, one), 0 * a.abs(), 0 * a.abs()
    z = a.abs()
    if name in ("silu", "sigmoid"):
        q, p = torch.sigmoid(a), torch.sigmoid(-a)
        rel = (z + 12) * U
        if name == "sigmoid":
            return q, q * p, rel * q + TINY, 2 * rel * q * p + TINY
        return a * q, q + a * q * p, rel * (a * q).abs() + TINY, 3 * rel * (q + z * q * p) + TINY
    if name == "gelu":
        cdf, pdf = 0.5 * torch.special.erfc(-a * math.sqrt(0.5)), torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
        rel = (3 * a * a + 50) * U
        return a * cdf, cdf + a * pdf, rel * (a * cdf).abs() + TINY, rel * (cdf + z * pdf) + TINY
    k = math.sqrt(2 / math.pi)
    u2, inner = 2 * k * (a + 0.044715 * a ** 3), 2 * k * (1 + 3 * 0.044715 * a * a)
    q, p = torch.sigmoid(u2), torch.sigmoid(-u2)
    rel = (6 * u2.abs() + 30) * U
    return a * q, q + a * q * p * inner, rel * (a * q).abs() + TINY, 2 * rel * (q + z * q * p * inner) + TINY


def gated_forward(x, wg, wu, bg, bu, act, dtype):
    """(m, gate, up) and their bounds."""
    cols = x.shape[1]
    a, b = x @ wg.t() + bg, x @ wu.t() + bu
    off_a = sums(x, wg.t(), cols) + 2 * U * (a.abs() + bg.abs())
    off_b = sums(x, wu.t(), cols) + 2 * U * (b.abs() + bu.abs())
    v, _, off_v, _ = activation(a, act)
    off_v = off_v + 1.2 * off_a       # no activation's slope is beyond 1.13
    m = v * b
    off_m = off_v * b.abs() + v.abs() * off_b + off_v * off_b + U * m.abs()
    more = 1 + UNIT[dtype]
    return (m, a, b), (rounding(m, dtype) + more * off_m, rounding(a, dtype) + more * off_a, rounding(b, dtype) + more * off_b)


def gated_backward(dm, a, b, n, act, dtype):
    """(dgate, dup, dgate_bias, dup_bias) and their bounds."""
    v, s, off_v, off_s = activation(a, act)
    dg, du = dm * b * s, dm * v
    off_g, off_u = (dm * b).abs() * (1.01 * off_s) + 3 * U * dg.abs() + TINY, dm.abs() * (1.01 * off_v) + 2 * U * du.abs() + TINY
    rows = dm.shape[0] // n
    by = lambda t: t.reshape(n, rows, -1).sum(1)  # noqa: E731
    # eight rows of a lane, up to 256 lanes, then the parts
    adds = 300 + rows / 8
    bounds = (rounding(dg, dtype) + 1.01 * off_g, rounding(du, dtype) + 1.01 * off_u,
              adds * U * by(dg.abs()) + by(off_g), adds * U * by(du.abs()) + by(off_u))
    return (dg, du, by(dg), by(du)), bounds


def projections(dgs, x, ws, n, dtype):
    """(dx, the weights' gradients) and their bounds, for one projection or two."""
    total = x.shape[0]
    rows = total // n
    dx = sum(d @ w for d, w in zip(dgs, ws))
    off = sum(sums(d, w, len(dgs) * d.shape[1]) for d, w in zip(dgs, ws))
    of = lambda t, i: t[i * rows:(i + 1) * rows]  # noqa: E731
    dw = [torch.stack([of(d, i).t() @ of(x, i) for i in range(n)]) for d in dgs]
    off_w = [torch.stack([sums(of(d, i).t(), of(x, i), rows) for i in range(n)]) + LEAST[torch.float32] for d in dgs]
    return [dx] + dw, [rounding(dx, dtype) + 1.01 * off] + off_w


def linear_cross_entropy(x, w, targets, n, ignore, grad_scale, dtype):
    """(mean_loss, losses, dx, dweight) and their bounds; targets that are no row of w give NaN."""
    total, cols = x.shape
    vocab, rows = w.shape[0], total // n
    learnt = targets != ignore
    x = torch.where(learnt[:, None], x, 0.0)      # ignored rows hold whatever they hold
    inside = (targets >= 0) & (targets < vocab)
    logits = x @ w.t()
    off_l = sums(x, w.t(), cols)
    top = torch.where(torch.isnan(logits).any(1, keepdim=True), torch.nan, logits.amax(1, keepdim=True))
    away = top - logits
    e = torch.exp(-away)
    s = e.sum(1, keepdim=True)
    at = torch.where(inside, targets, torch.zeros_like(targets))[:, None]
    of_target = logits.gather(1, at)
    loss = torch.where(inside[:, None], torch.log(s) + top - of_target, torch.nan)[:, 0]
    loss = torch.where(learnt, loss, 0.0)
    count = learnt.reshape(n, rows).sum(1).double()
    mean = torch.where(count > 0, loss.reshape(n, rows).sum(1) / count.clamp(min=1), 0.0)
    factor = torch.where(count > 0, grad_scale / count.clamp(min=1), 0.0)
    f = factor.repeat_interleave(rows)[:, None]
    hot = torch.zeros_like(logits).scatter_(1, at, 1.0)
    d = torch.where(inside[:, None], e / s - hot, torch.nan)
    d = torch.where(learnt[:, None], d, 0.0)
    finite = lambda t: torch.nan_to_num(t, nan=0.0, posinf=0.0, neginf=0.0)  # noqa: E731
    # the sum of the exponentials: 64 of a span as a tree of chains, the spans in sixteen chains, each rescaled at every span;
    # the weights' mean distance to the maximum is at most log V + 1
    spans = -(-vocab // 64)
    off_s = U * (60 + 8 * (spans / 16 + 16) + 4 * math.log(vocab + 1)) + 2 * finite(off_l).amax(1, keepdim=True)
    off_loss = off_s[:, 0] + 2 * finite(off_l).amax(1) + 4 * U * (finite(top[:, 0]).abs() + finite(of_target[:, 0]).abs()
                                                                  + finite(loss).abs() + 1)
    p = finite(e / s)
    off_d = p * (off_s + 4 * U * (finite(away) + 3) + 2 * finite(off_l)) + 4 * U * (p + hot) + 2.0 ** -140
    fd = finite(d)
    dx = (d * f) @ w
    # dx takes d rounded to its type; float16 holds 2^14 d
    held = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype] * fd.abs() + 2.0 ** -38
    off_x = f.abs() * ((off_d + held) @ w.abs() + sums(fd, w, vocab) + 4 * U * (fd.abs() @ w.abs()))
    of = lambda t, i: t[i * rows:(i + 1) * rows]  # noqa: E731
    dw = torch.stack([factor[i] * (of(d, i).t() @ of(x, i)) for i in range(n)])
    # d in parts: 2^-22 of each entry, or 2^-38 of the largest
    parts = 2.0 ** -22 * fd.abs() + 2.0 ** -38
    off_w = torch.stack([factor[i].abs() * (of(off_d + parts, i).t() @ of(x, i).abs() + sums(of(fd, i).t(), of(x, i), 3 * rows))
                         for i in range(n)])
    dx = torch.where(learnt[:, None], dx, 0.0)
    bounds = (off_loss.reshape(n, rows).amax(1) + 200 * U * finite(loss).abs().reshape(n, rows).sum(1) / count.clamp(min=1),
              off_loss, rounding(finite(dx), dtype) + 1.01 * torch.where(learnt[:, None], off_x, 0.0) + LEAST[dtype],
              off_w + 3 * U * finite(dw).abs() + 2.0 ** -140)
    return (mean, loss, dx, dw), bounds
