"""How many of their digits the operators keep, where an order of evaluation or a short cut could cost some: bounds that
follow from the rounding of each value by itself, for inputs on which the rest is exact or nearly so."""
import math

import numpy as np
import pytest
import torch

import operator_reference as R
from paper_2205_05632_amd import operators as ops

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
U = R.U


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [5, 300, 1500, 20000, 140000])
@pytest.mark.parametrize("rows", [19, 40])
def test_losses_do_not_depend_on_an_offset(rows, vocab, dtype):
    """What a row's logits have in common leaves its loss alone: log(sum exp(l - max)) + (max - target), where the sum is
    off by the reference's share of itself, the logarithm by two units, the difference and the sum by half a unit each."""
    tops = [0.0, 20.0, -100.0, 1e3, 3e4, -6e4] if dtype is F16 else \
        [0.0, 20.0, -100.0, 1e3, 1e4, -1e5, 1e6, -1e7, 1e9, -1e20, 1e30, 3e38]
    rng = np.random.default_rng(vocab + rows)
    v = rng.standard_normal((rows, vocab)) * 1.5
    t = torch.from_numpy(rng.integers(0, vocab, rows))
    v[::2, :] -= 3.0 * (np.arange(vocab)[None] != t.numpy()[::2, None])     # every other target well above the rest
    v = torch.from_numpy(v + np.resize(tops, rows)[:, None]).to(dtype)
    mean, losses, _ = ops.compams_cross_entropy(v.cuda(), t.cuda(), 1)
    v = v.double()
    away = v.amax(1) - v.gather(1, t[:, None])[:, 0]
    log_sum = torch.log(torch.exp(v - v.amax(1, keepdim=True)).sum(1))
    want = log_sum + away
    bound = 1.01 * U * (160 + 4 * math.log(vocab + 1) + 4 * log_sum + away + want)
    R.close(losses, want, bound, "losses")
    # (the mean: the losses' own errors, a sum of at most `rows` terms and a quotient)
    R.close(mean, want.mean(0, keepdim=True), bound.mean(0, keepdim=True) + 1.01 * U * (rows + 1) * want.mean(0, keepdim=True), "mean")
