"""The operators of the workers' models from their formulas in 64 bits, on the host, with the error that 32-bit arithmetic
may make in each entry.

Bounds.  U = 2^-24 is the unit roundoff of fp32, `unit(T)` that of the output's type T.  A sum of N terms of which a lane
adds at most 100 one after another and the rest as a tree is off by at most 128 U times the sum of the magnitudes; the
column sums (up to 64 rows or eight sixteenths of them one after another, then the parts) by at most 256 U times that.
Each output is then rounded once: unit(T) times its magnitude, and half the least denormal of float16.
"""
import math

import numpy as np
import torch

U = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def philox(counter, key):
    """Philox-4x32-10 on Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def numbers(rows, cols, seed, offset, first_row=0):
    """u(r, c) of a matrix, as numpy."""
    blocks = -(-cols // 8)
    m, h = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [np.broadcast_to(np.arange(blocks, dtype=np.uint64)[None], (rows, blocks)),
         np.broadcast_to(np.arange(first_row, first_row + rows, dtype=np.uint64)[:, None], (rows, blocks)),
         np.full((rows, blocks), offset & 0xFFFFFFFF, dtype=np.uint64),
         np.full((rows, blocks), (offset >> 32) & 0xFFFFFFFF, dtype=np.uint64)]
    k = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> h) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> h) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    u = np.empty((rows, blocks, 8), dtype=np.int64)
    for j in range(8):
        u[:, :, j] = (c[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF)
    return u.reshape(rows, 8 * blocks)[:, :cols]


def threshold(p):
    return math.floor(p * 65536 + 0.5)


def kept(rows, cols, p, seed, offset):
    return torch.from_numpy(numbers(rows, cols, seed, offset % 2 ** 64) >= threshold(p))


def factor(p):
    return 0.0 if threshold(p) == 65536 else 65536.0 / (65536 - threshold(p))


def rounding(value, dtype):
    return UNIT[dtype] * value.abs() + LEAST[dtype]


def close(got, want, bound, what):
    """Every entry of `got` within `bound` of `want`; what is not finite is the same on both sides."""
    got, want, bound = got.detach().cpu().double(), want.double(), bound.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    strange = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(got[strange].nan_to_num(nan=0.0), want[strange].nan_to_num(nan=0.0)), f"{what}: infinities differ"
    off = (got - want).abs()
    bad = ~strange & ~(off <= bound)
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} entries are off, by up to "
                                 f"{float((off / bound)[bad].max()):.3g} times the bound, first at "
                                 f"{tuple(int(i) for i in bad.nonzero()[0])}: {float(got[bad][0])} for {float(want[bad][0])}")


def norm_forward(h, gamma, beta, eps, dtype):
    """y, mean, rstd and their bounds, of h in 64 bits (exact, or with the error `h_off`)."""
    cols = h.shape[1]
    mean = h.sum(1) / cols
    d = h - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).sum(1) / cols + eps)
    z = d * rstd[:, None]
    size = h.abs().amax(1)
    y = z * gamma + beta
    a = (size * rstd)[:, None]
    off_z = 140 * U * (a + z.abs() * (a + 1.0))
    bounds = (rounding(y, dtype) + (1 + UNIT[dtype]) * (gamma.abs() * off_z + 4 * U * (y.abs() + beta.abs())),
              140 * U * size + U * mean.abs(), rstd * 140 * U * (size * rstd + 2.0))
    return (y, mean, rstd), bounds


def norm_backward(dy, dh, h, mean, rstd, gamma, stream_dtype, dtype, n, keep=None, scale=1.0):
    """(dx, dresidual, dgamma, dbeta, dbias) and their bounds, for the statistics as given."""
    total, cols = h.shape
    r = rstd[:, None]
    z = (h - mean[:, None]) * r
    u = dy * gamma
    s1, s2 = u.sum(1, keepdim=True) / cols, (u * z).sum(1, keepdim=True) / cols
    d = r * (u - s1 - z * s2)
    off = 140 * U * r * (u.abs() + u.abs().mean(1, keepdim=True) + 2 * z.abs() * (u * z).abs().mean(1, keepdim=True))
    if dh is not None:
        d = d + dh
        off = off + 2 * U * (d.abs() + dh.abs())
    dx, off_x = d, off
    if keep is not None:
        dx = torch.where(keep, d * scale, torch.zeros_like(d))
        off_x = torch.where(keep, off * scale + 2 * U * dx.abs(), torch.zeros_like(d))
    by = lambda t: t.reshape(n, total // n, cols).sum(1)  # noqa: E731
    values = (dx, d, by(dy * z), by(dy), by(dx))
    bounds = (rounding(dx, dtype) + 1.01 * off_x, rounding(d, stream_dtype) + 1.01 * off,
              260 * U * by((dy * z).abs()) + LEAST[torch.float32], 256 * U * by(dy.abs()) + LEAST[torch.float32],
              256 * U * by(dx.abs()) + by(off_x) + LEAST[torch.float32])
    return values, bounds


def cross_entropy(logits, targets, n, ignore, grad_scale, dtype):
    """(mean_loss, losses, dlogits) and their bounds; targets that are no column give NaN."""
    total, vocab = logits.shape
    rows = total // n
    learnt = targets != ignore
    inside = (targets >= 0) & (targets < vocab)
    top = logits.amax(1, keepdim=True)
    top = torch.where(torch.isnan(logits).any(1, keepdim=True), torch.nan, top)
    away = top - logits
    e = torch.exp(-away)
    s = e.sum(1, keepdim=True)
    at = torch.where(inside, targets, torch.zeros_like(targets))[:, None]
    of_target = logits.gather(1, at)
    loss = torch.where(inside[:, None], torch.log(s) + top - of_target, torch.nan)[:, 0]
    loss = torch.where(learnt, loss, 0.0)
    count = learnt.reshape(n, rows).sum(1).double()
    mean = torch.where(count > 0, loss.reshape(n, rows).sum(1) / count.clamp(min=1), 0.0)
    f = torch.where(learnt, grad_scale / count.repeat_interleave(rows).clamp(min=1), 0.0)[:, None]
    hot = torch.zeros_like(logits).scatter_(1, at, 1.0)
    d = torch.where(inside[:, None], (e / s - hot) * f, torch.nan)
    d = torch.where(learnt[:, None], d, 0.0)
    # exp: two units of its result and of its argument; the sum: 128 U, and the weights' mean argument is at most log V + 1
    finite = lambda t: torch.nan_to_num(t, nan=0.0, posinf=0.0, neginf=0.0)  # noqa: E731
    off_s = U * (160 + 4 * math.log(vocab + 1))
    off_loss = off_s + 4 * U * (finite(top[:, 0]).abs() + finite(of_target[:, 0]).abs() + finite(loss).abs() + 1)
    off_d = f.abs() * (finite(e / s) * (off_s + 4 * U * (finite(away) + 2)) + 4 * U * hot)
    bounds = (off_loss.reshape(n, rows).amax(1) + 160 * U * finite(loss).abs().reshape(n, rows).sum(1) / count.clamp(min=1),
              off_loss, rounding(finite(d), dtype) + 1.01 * off_d + 2.0 ** -140)
    return (mean, loss, d), bounds
