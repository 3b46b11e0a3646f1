"""Long sums of fp32 products, on the GPU against 64 bits: their error does not grow as that of a sum added up term by term.

A sum of K random terms that is added up one after another is off by U sqrt(K / 6) of itself (each addition by up to half a step of what is
there so far, evenly spread); in blocks of 64 that are added up in turn by U sqrt((64 + K / 64) / 6), and the products by U / sqrt(3).
Three times that is allowed, for what the matrix cores add within an instruction.  (Term by term, K = 16000 is at seven times.)"""
import math

import pytest
import torch

from operator_reference import U
from paper_2205_05632_amd import operators as ops

pytestmark = pytest.mark.gpu


def allowed(terms):
    return 3 * U * math.sqrt((64 + terms / 64) / 6 + 1 / 3)


def relative(got, want):
    return float((got.double() - want).norm() / want.norm())


def make(seed, *shapes):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(s, generator=g, device="cuda") for s in shapes]


@pytest.mark.parametrize("rows,cols,hidden", [(16000, 72, 40), (9001, 300, 520)])
def test_weights_gradients_of_many_rows(rows, cols, hidden):
    x, dg, du = make(rows, (rows, cols), (rows, hidden), (rows, hidden))
    _, a, b = ops.compams_projections_backward(dg, du, x, None, None, 1)
    assert relative(a, dg.double().t() @ x.double()) < allowed(rows) and relative(b, du.double().t() @ x.double()) < allowed(rows)


@pytest.mark.parametrize("rows,cols,hidden", [(100, 4000, 130), (2000, 8003, 1500)])
def test_projections_of_wide_rows(rows, cols, hidden):
    x, wg, wu = make(rows, (rows, cols), (hidden, cols), (hidden, cols))
    _, a, b = ops.compams_gated_forward(x, wg, wu, "relu")
    assert relative(a, x.double() @ wg.double().t()) < allowed(cols) and relative(b, x.double() @ wu.double().t()) < allowed(cols)


@pytest.mark.parametrize("rows,cols,hidden", [(3000, 500, 6000)])
def test_dx_of_wide_blocks(rows, cols, hidden):
    dg, du, wg, wu = make(rows, (rows, hidden), (rows, hidden), (hidden, cols), (hidden, cols))
    dx = ops.compams_projections_backward(dg, du, None, wg, wu, 1)[0]
    assert relative(dx, dg.double() @ wg.double() + du.double() @ wu.double()) < allowed(2 * hidden)


def test_output_layer():
    """The weight's gradient of many rows, and dx over a vocabulary of several pieces.  (x is small, so that the logits' errors are.)"""
    rows, cols, vocab = 9000, 48, 5000
    x, w = make(1, (rows, cols), (vocab, cols))
    x *= 1e-3
    t = torch.randint(0, vocab, (rows,), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    _, _, dx, dw = ops.compams_linear_cross_entropy(x, w, t, 1, -100, float(rows))
    d = torch.softmax(x.double() @ w.double().t(), 1)
    d[torch.arange(rows), t] -= 1
    # (an entry of d is off by its exponential and 1 / sum: 4 U of a probability, 1 / vocab, beside the target's 1)
    assert relative(dw, d.t() @ x.double()) < allowed(rows) + 4 * U and relative(dx, d @ w.double()) < allowed(vocab) + 4 * U
