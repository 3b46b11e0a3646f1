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


ROUTES = [(1, 24), (40, 24), (1, 500), (700, 130), (3, 2000), (40, 5000), (40, 20000), (3, 140000)]    # (rows of one worker, columns)


def few_entries(rng, rows, vocab, dtype, far):
    """Rows of minus infinity but for six entries: the largest, 0, and five at whole and half distances up to `far` below, so
    that every difference is exact and a row's sum has six terms.  (logits, targets: the largest or another of the six)"""
    at = torch.from_numpy(np.stack([rng.choice(vocab, 6, replace=False) for _ in range(rows)]))
    away = torch.from_numpy(rng.integers(0, 2 * far, (rows, 6)) / 2.0)
    away[:, 0] = 0.0
    v = torch.full((rows, vocab), -math.inf, dtype=torch.float64).scatter_(1, at, -away)
    t = at[:, 0].clone()
    t[1::3] = at[1::3, 1]
    return v.to(dtype), t


def gradient_of(v, t, scale):
    """(gradient, probabilities, where the targets are), in 64 bits."""
    p = torch.softmax(v.double(), 1)
    hot = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    return (p - hot) * scale, p, hot


@pytest.mark.parametrize("rows,vocab", ROUTES)
def test_exponentials_at_every_distance(rows, vocab):
    """Entries of fp32 rows keep their digits at any distance to the row's maximum: an exponential four units, the sum of six
    of them those and six roundings, the quotient and the product one each."""
    v, t = few_entries(np.random.default_rng(rows + vocab), rows, vocab, F32, 100)
    _, _, d = ops.compams_cross_entropy(v.cuda(), t.cuda(), 1, grad_scale=float(rows))
    want, p, hot = gradient_of(v, t, 1.0)
    R.close(d, want, 16 * U * p + 2 * U * hot + 2.0 ** -149, "dlogits")


@pytest.mark.parametrize("dtype,scale", [(F32, 2.0 ** 15), (F32, -3.0 * 2.0 ** 40), (F32, 2.0 ** 110), (F16, 2.0 ** 15),
                                         (BF16, 2.0 ** 15), (BF16, -3.0 * 2.0 ** 40), (BF16, 2.0 ** 110)],
                         ids=["f32_15", "f32_41", "f32_110", "f16_15", "bf16_15", "bf16_41", "bf16_110"])
@pytest.mark.parametrize("rows,vocab", ROUTES)
def test_what_a_scale_brings_back(rows, vocab, dtype, scale):
    """Of a scaled loss the gradient, not the probability, decides what is too small to be held, with scales up to 2^96 at
    least.  (Of 16 bits an exponential is off by 2.3 units for each of the distance and two for each power of two of the
    scale, and subnormal results may be 0.)"""
    v, t = few_entries(np.random.default_rng(rows + vocab + 1), rows, vocab, dtype, 115)
    _, _, d = ops.compams_cross_entropy(v.cuda(), t.cuda(), 1, grad_scale=scale * rows)
    want, p, hot = gradient_of(v, t, scale)
    units, least = 16.0, 2.0 ** -149
    if dtype is not F32:
        units, least = 16.0 + 2.3 * (-v.double()).clamp(max=200.0) + 2 * math.log2(abs(scale) * rows), 2.0 ** -126 + R.LEAST[dtype]
    least = max(least, 2.0 ** -125 * abs(scale) / 2.0 ** 96)
    R.close(d, want, (units * U * p + 2 * U * hot) * abs(scale) + R.UNIT[dtype] * 1.01 * want.abs() + least, "dlogits")


@pytest.mark.parametrize("join", [False, True], ids=["norm", "join"])
@pytest.mark.parametrize("cols", [6, 10, 24, 100, 333, 768, 1000, 1601, 2304, 6144, 10484, 12288, 20000, 33000])
def test_statistics_are_rounded_once(cols, join):
    """Rows of whole numbers, whose sums are exact: the mean is the quotient to the nearest, on every route the same; where
    the mean is whole the sum of squares is exact too, and rstd what correct rounding makes of the quotient and of eps
    added, and then of the inverse root (half a unit in its last place, and a 64th for the residual's own rounding)."""
    rng = np.random.default_rng(cols)
    rows = 24
    v = rng.integers(-20, 21, (rows, cols)).astype(np.float64)
    short = (-v.sum(1)) % cols * (np.arange(rows) % 2)       # every other row: a whole mean
    v += np.arange(cols)[None] < short[:, None]
    x = torch.from_numpy(v).float().cuda()
    if join:
        _, _, mean, rstd = ops.compams_dropout_add_norm_forward(torch.zeros_like(x), x, None, None, 0.0, 1, eps=0.25)
    else:
        _, mean, rstd = ops.compams_layer_norm_forward(x, None, None, 0.25)
    assert np.array_equal(mean.cpu().numpy(), np.float32(v.sum(1)) / np.float32(cols))
    whole = v[1::2]
    squares = ((whole - whole.mean(1, keepdims=True)) ** 2).sum(1)
    assert squares.max() < 2 ** 24
    var = (np.float32(squares) / np.float32(cols) + np.float32(0.25)).astype(np.float64)
    got = rstd[1::2].cpu().numpy()
    assert np.all(np.abs(got.astype(np.float64) - var ** -0.5) <= (0.5 + 1 / 64) * np.spacing(got))


@pytest.mark.parametrize("whole", [False, True], ids=["without_gamma", "with_gamma"])
@pytest.mark.parametrize("join", [False, True], ids=["norm", "join"])
@pytest.mark.parametrize("cols", [3, 7, 9, 72, 100, 333, 776, 1000, 1601, 2056, 2500, 6000, 6001, 9000, 20001])
def test_gradients_of_equal_entries_of_any_size(cols, join, whole):
    """Rows whose entries are all the same have z = 0 and a gradient of rstd (u - mean u), however large the entries are: what
    stands beside the row's columns in a lane has no part in its sums."""
    rng = np.random.default_rng(cols)
    rows = 9
    size = np.float32(10.0) ** np.linspace(0, 38, rows, dtype=np.float32)
    x = torch.from_numpy(size)[:, None].expand(rows, cols).contiguous().cuda()
    mean, rstd = torch.from_numpy(size).cuda(), torch.full((rows,), 300.0, device="cuda")
    dy = torch.from_numpy(rng.standard_normal((rows, cols))).float()
    one, gamma = torch.ones(cols), torch.ones(cols, device="cuda") if whole else None
    if join:
        dh = torch.zeros_like(x) if whole else None
        _, dx, dgamma, dbeta, _ = ops.compams_dropout_add_norm_backward(dy.cuda(), dh, x, mean, rstd, gamma, 0.0, 1)
    else:
        dx, dgamma, dbeta = ops.compams_layer_norm_backward(dy.cuda(), x, mean, rstd, gamma)
    want, bound = R.norm_backward(dy.double(), None, x.cpu().double(), mean.cpu().double(), rstd.cpu().double(), one.double(),
                                  F32, F32, 1)
    R.close(dx, want[1], bound[1], "dx")
    R.close(dgamma, want[2], bound[2], "dgamma")
    R.close(dbeta, want[3], bound[3], "dbeta")
