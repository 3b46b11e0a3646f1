"""The digits that the output layer's cross-entropy keeps, on the GPU against the formulas in 64 bits."""
import math

import numpy as np
import pytest
import torch

import product_reference as P
from operator_reference import LEAST, U, close, rounding
from paper_2205_05632_amd import operators as ops

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
IDS = ["f32", "f16", "bf16"]


def gradients(x, w, t, n, grad_scale, dtype):
    """(dx, dweight) and their bounds where no row is ignored.  A probability p is off by its logit's error and its maximum's, by the
    sum of the exponentials (64 of a span, the spans in chains) and by 4 U (z + 3) at a distance z; d by that and 4 U.  16 bits: two
    parts of 2^14 d hold it to 2^-22 of itself or 2^-38, and an entry of bfloat16's operands is off by 2^-38 of its column's largest.
    Both sums go once through their terms for each part."""
    total, cols = x.shape
    vocab, rows, parts = w.shape[0], total // n, 1 if dtype == F32 else 2
    logits = x @ w.t()
    off_l = P.sums(x, w.t(), cols)
    away = logits.amax(1, keepdim=True) - logits
    p = torch.softmax(logits, 1)
    hot = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    d = p - hot
    off_s = U * (60 + 8 * (-(-vocab // 64) / 16 + 16) + 4 * math.log(vocab + 1)) + 2 * off_l.amax(1, keepdim=True)
    off_d = p * (off_s + 4 * U * (away + 3) + 2 * off_l) + 4 * U * (p + hot) + 2.0 ** -140
    if parts == 2:
        off_d = off_d + 2.0 ** -22 * d.abs() + 2.0 ** -38
    f, lost = grad_scale / rows, 2.0 ** -38 if dtype == BF16 else 0.0

    def product(off, a, b, terms):
        return f * (off @ b.abs() + P.sums(a, b, parts * terms) + 4 * U * (a.abs() @ b.abs()) + lost * b.abs().amax(0) * a.abs().sum(1, keepdim=True))

    dx = f * (d @ w)
    of = lambda v, i: v[i * rows:(i + 1) * rows]  # noqa: E731
    dw = torch.stack([f * (of(d, i).t() @ of(x, i)) for i in range(n)])
    off_w = torch.stack([product(of(off_d, i).t(), of(d, i).t(), of(x, i), rows) for i in range(n)])
    return (dx, dw), (rounding(dx, dtype) + 1.01 * product(off_d, d, w, vocab) + LEAST[dtype], off_w + U * dw.abs() + 2.0 ** -140)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,rows,cols,vocab", [(2, 33, 8, 32), (1, 100, 16, 64), (3, 20, 40, 300), (1, 300, 24, 1100), (1, 9, 16, 5000)])
def test_gradients_have_the_digits_of_fp32(n, rows, cols, vocab, dtype):
    """Every entry of dx is rounded once, and what it is rounded from has fp32's error: in columns whose terms cancel it shows.  (A
    gradient's entries add up to 0, so the first column's is 0: its weights are all 1.)"""
    rng = np.random.default_rng(vocab)
    make = lambda r, c, s: torch.from_numpy(rng.standard_normal((r, c)) * s).to(dtype)  # noqa: E731
    x, w = make(n * rows, cols, 1.0), make(vocab, cols, 1.0 / math.sqrt(cols))
    x[:, 0], w[:, 0] = 0.0, 1.0
    w[:, 1] = (1.0 + w[:, 1].float() / 64).to(dtype)
    t = torch.from_numpy(rng.integers(0, vocab, n * rows))
    got = ops.compams_linear_cross_entropy(x.cuda(), w.cuda(), t.cuda(), n, -100, float(rows))[2:]
    for g, want, bound, what in zip(got, *gradients(x.double(), w.double(), t, n, float(rows), dtype), ("dx", "dweight")):
        close(g, want, bound, what)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,rows,cols,vocab", [(2, 9000, 40, 4100), (8, 5000, 16, 1100), (4, 512, 256, 5000)])
def test_dx_of_several_pieces_has_the_digits_of_fp32(n, rows, cols, vocab, dtype):
    """The first column of dx, whose terms cancel, at sizes that take several pieces of the vocabulary, large tiles or parts."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn((n * rows, cols), generator=g, device="cuda").to(dtype)
    w = (torch.randn((vocab, cols), generator=g, device="cuda") * 2.5 / math.sqrt(cols)).to(dtype)
    x[:, 0], w[:, 0] = 0.0, 1.0
    t = torch.randint(0, vocab, (n * rows,), generator=g, device="cuda")
    dx = ops.compams_linear_cross_entropy(x, w, t, n, -100, float(rows))[2]
    # A sum of K random terms is off by about U sqrt(K / 2) of its own size, twice that where sums are cut; 4 U sqrt(K) leaves a factor of
    # three (of the norm; five times that for the largest of all rows).  The size is that of d's two signs, 1 each; logits of size 3.
    off = 4 * U * math.sqrt(2 * vocab) + 4 * U * math.sqrt(cols) * 3 + 200 * U + 2.0 ** -22
    column = dx[:, 0].double()
    assert float(column.norm()) < off * math.sqrt(n * rows) and float(column.abs().max()) < 5 * off


@pytest.mark.parametrize("n,vocab", [(3, 8), (4, 40), (2, 130), (70, 300)])
def test_far_entries_of_fp32_keep_their_digits(n, vocab):
    """Probabilities down to e^-80: exact to some units of fp32 however far their logits are.  (The weight is the unit matrix and the
    logits are eighths, so that neither they nor their distances are rounded; a row to a worker.)"""
    g = torch.Generator().manual_seed(vocab)
    x = -torch.randint(160, 641, (n, vocab), generator=g).double() / 8
    x[:, 3] = 0.0
    t = torch.randint(0, vocab, (n,), generator=g)
    t[0] = 3
    got = ops.compams_linear_cross_entropy(x.float().cuda(), torch.eye(vocab, device="cuda"), t.cuda(), n)
    p = torch.softmax(x, 1)
    hot = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    d = p - hot
    # an exponential 3 U, 1 / sum (1 and terms below e^-20) 3 U, products with that, the factor and x U each; next to the target's 1
    # the difference is rounded, and a difference of 0 may have all of p's errors
    off = 10 * U * p + 2 * U * hot
    close(got[2], d, off, "dx")
    close(got[3], d[:, :, None] * x[:, None, :], (off + U * d.abs())[:, :, None] * x.abs()[:, None, :], "dweight")
    want = torch.logsumexp(x, 1) - x.gather(1, t[:, None])[:, 0]
    close(got[1], want, 2 * U * want.abs() + 4 * U * p.sort(1).values[:, :-1].sum(1) + 2 * U * (p.sort(1).values[:, :-1].sum(1) > 0), "losses")
