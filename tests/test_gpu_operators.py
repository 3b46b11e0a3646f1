"""The operators of the workers' models on the GPU against their formulas in 64 bits."""
import ctypes
import math

import numpy as np
import pytest
import torch

import operator_reference as R
from paper_2205_05632_amd import binding as B
from paper_2205_05632_amd import operators as ops

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)]    # (branch, stream)
IDS = ["f32", "f16", "bf16", "f16_f32", "bf16_f32"]
EPS = 1e-5


def matrix(rng, total, cols, dtype, pad=0, shift=0, scale=1.0):
    """A matrix on the GPU whose rows are `pad` columns apart and start `shift` columns after the allocation, and its
    values in 64 bits; what lies around the rows is NaN."""
    v = torch.from_numpy(rng.standard_normal((total, cols)) * scale).to(dtype)
    base = torch.full((total, cols + pad + shift), math.nan, dtype=dtype, device="cuda")
    base[:, shift:shift + cols] = v.cuda()
    return base[:, shift:shift + cols], v.double()


def room(total, cols, dtype, pad=0, shift=0, fill=7.0):
    base = torch.full((total, cols + pad + shift), fill, dtype=dtype, device="cuda")
    return base[:, shift:shift + cols], base


def untouched(base, shift, cols, fill=7.0):
    assert bool((base[:, :shift] == fill).all()) and bool((base[:, shift + cols:] == fill).all())


def vector(rng, cols, around=0.0, shift=0):
    v = torch.from_numpy(rng.standard_normal(cols) * 0.3 + around).float()
    base = torch.full((cols + shift,), math.nan, device="cuda")
    base[shift:] = v.cuda()
    return base[shift:], v.double()


WIDTHS = [1, 2, 7, 8, 9, 63, 64, 65, 127, 128, 250, 256, 257, 513, 768, 1000, 1024, 1025, 1600, 2048, 2049, 4096, 4099, 8192,
          8200, 12289, 16385, 32768, 40001]


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("cols", WIDTHS)
def test_layer_norm(cols, types):
    """Forward and backward, rows apart and starting anywhere; the odd widths with weights that start anywhere too."""
    dtype, stream = types
    rng = np.random.default_rng(cols * 8 + TYPES.index(types))
    n, rows = (3, 5) if cols > 4096 else (2, 37)
    pad, shift = (3, 1) if cols % 2 else (0, 0)
    x, x64 = matrix(rng, n * rows, cols, stream, pad, shift, 2.0)
    gamma, g64 = vector(rng, cols, 1.0, shift)
    beta, b64 = vector(rng, cols, 0.0, shift)
    y, ybase = room(n * rows, cols, dtype, pad, shift)
    y, mean, rstd = ops.compams_layer_norm_forward(x, gamma, beta, EPS, y=y)
    want, bound = R.norm_forward(x64, g64, b64, EPS, dtype)
    for got, w, b, what in zip((y, mean, rstd), want, bound, ("y", "mean", "rstd")):
        R.close(got, w, b, what)
    untouched(ybase, shift, cols)

    dy, dy64 = matrix(rng, n * rows, cols, dtype, pad, shift, 0.5)
    dx, xbase = room(n * rows, cols, stream, pad, shift)
    dx, dgamma, dbeta = ops.compams_layer_norm_backward(dy, x, mean, rstd, gamma, n, dx=dx)
    want, bound = R.norm_backward(dy64, None, x64, mean.cpu().double(), rstd.cpu().double(), g64, stream, dtype, n)
    R.close(dx, want[1], bound[1], "dx")
    R.close(dgamma, want[2], bound[2], "dgamma")
    R.close(dbeta, want[3], bound[3], "dbeta")
    untouched(xbase, shift, cols)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("cols", [1, 9, 64, 96, 250, 768, 1111, 1600, 2500, 4100, 9000, 33000])
def test_join(cols, types):
    """Bias, dropout, residual add and layer norm, and the gradient of all of it."""
    dtype, stream = types
    rng = np.random.default_rng(cols * 8 + TYPES.index(types) + 100000)
    n, rows = (2, 3) if cols > 4096 else (3, 21)
    pad, shift = (5, 3) if cols % 2 else (8, 0)
    p, seed, offset = 0.2, 0xFEDCBA9876543210 + cols, (7 << 32) + 11
    x, x64 = matrix(rng, n * rows, cols, dtype, pad, shift)
    res, r64 = matrix(rng, n * rows, cols, stream, pad, shift, 2.0)
    gamma, g64 = vector(rng, cols, 1.0, shift)
    beta, b64 = vector(rng, cols, 0.0, shift)
    bias, c64 = vector(rng, cols, 0.0, shift)
    h, hbase = room(n * rows, cols, stream, pad, shift)
    h, y, mean, rstd = ops.compams_dropout_add_norm_forward(x, res, gamma, beta, p, seed, offset, EPS, bias=bias, h=h)
    keep, scale = R.kept(n * rows, cols, p, seed, offset), R.factor(p)
    branch = torch.where(keep, (x64 + c64) * scale, torch.zeros_like(x64))
    h64 = r64 + branch
    off_h = 4 * R.U * (branch.abs() + h64.abs())
    R.close(h, h64, R.rounding(h64, stream) + 1.01 * off_h, "h")
    want, bound = R.norm_forward(h64, g64, b64, EPS, dtype)    # (h's own error of 4 U is within the 140 U of its bounds)
    for got, w, b, what in zip((y, mean, rstd), want, bound, ("y", "mean", "rstd")):
        R.close(got, w, b, what)
    untouched(hbase, shift, cols)

    dy, dy64 = matrix(rng, n * rows, cols, dtype, pad, shift, 0.5)
    dh, dh64 = matrix(rng, n * rows, cols, stream, pad, shift, 0.5)
    got = ops.compams_dropout_add_norm_backward(dy, dh, h, mean, rstd, gamma, p, seed, offset, n)
    want, bound = R.norm_backward(dy64, dh64, h.cpu().double(), mean.cpu().double(), rstd.cpu().double(), g64, stream, dtype, n,
                                  keep, scale)
    for g, w, b, what in zip(got, want, bound, ("dx", "dresidual", "dgamma", "dbeta", "dbias")):
        R.close(g, w, b, what)


@pytest.mark.parametrize("types", [(F32, F32), (BF16, F32)], ids=["f32", "bf16_f32"])
@pytest.mark.parametrize("cols", [3, 7, 8, 24, 128, 512, 640, 900, 1024, 1280, 1700, 2000, 2048, 8192, 8193, 12288, 13000, 16400])
def test_join_of_every_kind_of_team(cols, types):
    test_join(cols, types)


@pytest.mark.parametrize("n,rows,vocab", [(1, 32, 1000), (3, 32, 1000), (3, 33, 1000), (257, 4, 40), (2, 1, 2048), (5, 17, 500),
                                          (4, 100, 300), (1, 3000, 64), (2, 400, 90)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_cross_entropy_of_many_shapes(n, rows, vocab, dtype):
    """Few and many rows to a worker, among them workers that learn from none."""
    rng = np.random.default_rng(n * 100 + rows + vocab)
    x, x64 = matrix(rng, n * rows, vocab, dtype, 3, 1, 2.0)
    t = torch.from_numpy(rng.integers(0, vocab, n * rows))
    t[torch.from_numpy(rng.random(n * rows) < 0.3)] = -100
    t[(n - 1) * rows:] = -100
    got = ops.compams_cross_entropy(x, t.cuda(), n)
    want, bound = R.cross_entropy(x64, t, n, -100, 1.0, dtype)
    for g, w, b, what in zip(got, want, bound, ("mean_loss", "losses", "dlogits")):
        R.close(g, w, b, what)


@pytest.mark.parametrize("n,rows", [(1, 1), (5, 1), (2, 2), (1, 31), (2, 63), (2, 64), (2, 65), (3, 129), (1, 1000), (16, 300),
                                    (1, 4097), (300, 3)])
@pytest.mark.parametrize("cols", [24, 768, 2080])
def test_sums_over_any_number_of_rows(n, rows, cols):
    """The weights' gradients, into the workers' rows of a gradient buffer: first written, then added to."""
    if n * rows * cols > 4_000_000:
        cols = 24
    rng = np.random.default_rng(n * 7919 + rows * 31 + cols)
    x, x64 = matrix(rng, n * rows, cols, BF16)
    dy, dy64 = matrix(rng, n * rows, cols, BF16)
    dh, dh64 = matrix(rng, n * rows, cols, BF16)
    gamma, g64 = vector(rng, cols, 1.0)
    mean, rstd = vector(rng, n * rows)[0], vector(rng, n * rows, 1.0)[0]
    ld = 3 * cols + 10
    buf = torch.full((n, ld), math.nan, device="cuda")
    at = [buf[:, 1 + i * cols:1 + (i + 1) * cols] for i in range(3)]
    keep, p, seed = R.kept(n * rows, cols, 0.1, 5, 6), 0.1, 5
    kw = dict(dgamma=at[0], dbeta=at[1], dbias=at[2])
    first = ops.compams_dropout_add_norm_backward(dy, dh, x, mean, rstd, gamma, p, seed, 6, n, **kw)
    want, bound = R.norm_backward(dy64, dh64, x64, mean.cpu().double(), rstd.cpu().double(), g64, BF16, BF16, n, keep, R.factor(p))
    assert first[2].data_ptr() == at[0].data_ptr()
    for g, w, b, what in zip(at, want[2:], bound[2:], ("dgamma", "dbeta", "dbias")):
        R.close(g, w, b, what)
    once = [t.clone() for t in at]
    ops.compams_dropout_add_norm_backward(dy, dh, x, mean, rstd, gamma, p, seed, 6, n, accumulate=True, **kw)
    for a, b in zip(at, once):
        assert torch.equal(a, b + b)              # the same bits again, added to themselves
    assert bool(torch.isnan(buf[:, :1]).all()) and bool(torch.isnan(buf[:, 1 + 3 * cols:]).all())
    # a worker on its own gives the same bits, whatever stands beside it
    if n > 1:
        w = n - 1
        part = slice(w * rows, (w + 1) * rows)
        alone = ops.compams_layer_norm_backward(dy[part], x[part], mean[part], rstd[part], gamma, 1)
        beside = ops.compams_layer_norm_backward(dy, x, mean, rstd, gamma, n)
        assert torch.equal(alone[0], beside[0][part])
        assert torch.equal(alone[1][0], beside[1][w]) and torch.equal(alone[2][0], beside[2][w])


def test_weights_that_are_not_there_and_outputs_that_are_not_wanted():
    rng = np.random.default_rng(3)
    n, rows, cols = 2, 9, 200
    x, x64 = matrix(rng, n * rows, cols, F32)
    one, zero = torch.ones(cols).double(), torch.zeros(cols).double()
    y, mean, rstd = ops.compams_layer_norm_forward(x, None, None)
    want, bound = R.norm_forward(x64, one, zero, EPS, F32)
    R.close(y, want[0], bound[0], "y")
    # join without dropout, residual, bias and weights: the layer norm
    h, y2, mean2, rstd2 = ops.compams_dropout_add_norm_forward(x, None, None, None, 0.0, 1)
    assert torch.equal(h, x) and torch.equal(y, y2) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    dy, dy64 = matrix(rng, n * rows, cols, F32)
    full = ops.compams_dropout_add_norm_backward(dy, None, x, mean, rstd, None, 0.0, 1, 0, n)
    want, bound = R.norm_backward(dy64, None, x64, mean.cpu().double(), rstd.cpu().double(), one, F32, F32, n)
    for g, w, b in zip(full, want, bound):
        R.close(g, w, b, "a gradient without weights")
    names = ["dx", "dresidual", "dgamma", "dbeta", "dbias"]
    for wanted in (["dx"], ["dresidual"], ["dgamma"], ["dbeta"], ["dbias"], ["dx", "dbias"], ["dresidual", "dgamma", "dbeta"]):
        out = {k: torch.full_like(full[names.index(k)], 3.0) for k in wanted}
        a = ops.compams_norm(n=n, rows=rows, cols=cols, type=ops.F32, stream_type=ops.F32, h=x.data_ptr(), ld_h=cols,
                             mean=mean.data_ptr(), rstd=rstd.data_ptr(), dy=dy.data_ptr(), ld_dy=cols)
        for k, t in out.items():
            setattr(a, k, t.data_ptr())
            setattr(a, "ld_" + k, cols)
        ws = torch.empty(max(1, B.lib().compams_norm_workspace_size(ctypes.byref(a))), dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
        assert B.lib().compams_dropout_add_norm_backward(ctypes.byref(a), None) == 0
        torch.cuda.synchronize()
        for k, t in out.items():
            assert torch.equal(t, full[names.index(k)]), (wanted, k)
    # forward without statistics and without h
    out = torch.empty_like(x)
    a = ops.compams_norm(n=n, rows=rows, cols=cols, type=ops.F32, stream_type=ops.F32, eps=EPS, x=x.data_ptr(), ld_x=cols,
                         y=out.data_ptr(), ld_y=cols)
    assert B.lib().compams_dropout_add_norm_forward(ctypes.byref(a), None) == 0
    torch.cuda.synchronize()
    assert torch.equal(out, y)


@pytest.mark.parametrize("cols", [96, 1500, 6000, 34000])
def test_outputs_over_inputs(cols):
    """The outputs that may be an input's own buffer, on every route."""
    rng = np.random.default_rng(cols)
    n, rows, p, seed = 2, 6, 0.3, 9
    x, _ = matrix(rng, n * rows, cols, F32)
    res, _ = matrix(rng, n * rows, cols, F32)
    gamma, beta = vector(rng, cols, 1.0)[0], vector(rng, cols)[0]
    h, y, mean, rstd = ops.compams_dropout_add_norm_forward(x, res, gamma, beta, p, seed)
    x2, res2 = x.clone(), res.clone()
    ops.compams_dropout_add_norm_forward(x2, res2, gamma, beta, p, seed, h=res2, y=x2)
    assert torch.equal(res2, h) and torch.equal(x2, y)
    z = x.clone()
    ops.compams_layer_norm_forward(z, gamma, beta, y=z)
    assert torch.equal(z, ops.compams_layer_norm_forward(x, gamma, beta)[0])
    dy, _ = matrix(rng, n * rows, cols, F32)
    dh, _ = matrix(rng, n * rows, cols, F32)
    want = ops.compams_dropout_add_norm_backward(dy, dh, h, mean, rstd, gamma, p, seed, 0, n)
    dy2, dh2 = dy.clone(), dh.clone()
    got = ops.compams_dropout_add_norm_backward(dy2, dh2, h, mean, rstd, gamma, p, seed, 0, n, dx=dy2, dresidual=dh2)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    d = x.clone()
    assert torch.equal(ops.compams_dropout(d, p, seed, y=d), ops.compams_dropout(x, p, seed))
    d = res.clone()
    assert torch.equal(ops.compams_dropout(x, p, seed, residual=d, y=d), ops.compams_dropout(x, p, seed, residual=res))
    t = torch.from_numpy(rng.integers(0, cols, n * rows)).cuda()
    _, losses, dl = ops.compams_cross_entropy(x, t, n)
    over = x.clone()
    _, losses2, _ = ops.compams_cross_entropy(over, t, n, dlogits=over)
    assert torch.equal(over, dl) and torch.equal(losses, losses2)


def test_rows_that_a_norm_is_hard_on():
    """Constant rows, rows far from zero, rows with entries that are not finite."""
    rng = np.random.default_rng(8)
    for cols in (5, 768, 3000, 40000):
        v = rng.standard_normal((6, cols)) * 1e-3
        v[0] = 3.25
        v[1] += 1000.0
        v[2] *= 1e18
        v[3] *= 1e-30
        v = torch.from_numpy(v).float()
        v[4, cols // 2] = math.inf
        v[5, cols - 1] = math.nan
        y, mean, rstd = ops.compams_layer_norm_forward(v.cuda(), None, None)
        want, bound = R.norm_forward(v[:4].double(), torch.ones(cols).double(), torch.zeros(cols).double(), EPS, F32)
        for got, w, b, what in zip((y, mean, rstd), want, bound, ("y", "mean", "rstd")):
            R.close(got[:4], w, b, what)
        assert bool(torch.isnan(y[4:]).all()), cols
        # neighbours of such rows keep their values
        again = ops.compams_layer_norm_forward(v[:4].cuda().contiguous(), None, None)
        assert torch.equal(again[0], y[:4])


@pytest.mark.parametrize("kinds", [(F32, F32), (F16, F16), (BF16, BF16), (F32, F16), (F32, BF16), (F16, F32), (BF16, F32)],
                         ids=lambda k: f"{k[0]}_{k[1]}".replace("torch.", ""))
@pytest.mark.parametrize("total,cols", [(1, 1), (3, 7), (5, 8), (64, 50), (7, 768), (3, 2049), (2, 70001), (1000, 3)])
def test_dropout(total, cols, kinds):
    xt, yt = kinds
    rng = np.random.default_rng(total * 100 + cols)
    p, seed, offset = 0.35, 77 + cols, 2 ** 40 + 5
    keep = R.kept(total, cols, p, seed, offset)
    for pad, shift in ((0, 0), (5, 1)):
        x, x64 = matrix(rng, total, cols, xt, pad, shift)
        res, r64 = matrix(rng, total, cols, yt, pad, shift)
        y, base = room(total, cols, yt, pad, shift)
        ops.compams_dropout(x, p, seed, offset, y=y)
        want = torch.where(keep, x64 * R.factor(p), torch.zeros_like(x64))
        R.close(y, want, R.rounding(want, yt) + 2 * R.U * want.abs(), "y")
        assert torch.equal(y.cpu() != 0, keep & (x64 != 0))
        untouched(base, shift, cols)
        ops.compams_dropout(x, p, seed, offset, residual=res, y=y)
        R.close(y, want + r64, R.rounding(want + r64, yt) + 3 * R.U * (want.abs() + r64.abs()), "residual + y")
        untouched(base, shift, cols)


def test_dropout_edges():
    x = torch.randn(64, 1000, device="cuda")
    assert torch.equal(ops.compams_dropout(x, 0.0, 1), x)
    assert torch.equal(ops.compams_dropout(x, 1e-6, 1), x)               # less than half a 65536th
    y = ops.compams_dropout(torch.full_like(x, math.nan), 1.0, 1)
    assert torch.equal(y, torch.zeros_like(x))                           # whatever it was
    strange = torch.full_like(x, math.nan)
    strange[:, ::2] = math.inf
    keep = R.kept(64, 1000, 0.5, 3, 4)
    y = ops.compams_dropout(strange, 0.5, 3, 4).cpu()
    assert bool((y[~keep] == 0).all()) and bool(torch.isnan(y[:, 1::2][keep[:, 1::2]]).all())
    assert bool(torch.isinf(y[:, ::2][keep[:, ::2]]).all())
    # one at a time: seed and offset matter in all their bits, and rows are their own
    base = ops.compams_dropout(x, 0.5, 3, 4)
    for seed, offset in ((3 + 2 ** 63, 4), (3, 4 + 2 ** 63), (2, 4), (3, 5)):
        other = ops.compams_dropout(x, 0.5, seed, offset)
        assert not torch.equal(other, base)
        assert torch.equal(other.cpu() != 0, R.kept(64, 1000, 0.5, seed, offset) & (x.cpu() != 0))
    step = torch.tensor([-1], dtype=torch.int64, device="cuda")          # added modulo 2^64
    assert torch.equal(ops.compams_dropout(x, 0.5, 3, 5, step=step), base)
    # a share of p is dropped: 64 000 entries, five standard deviations
    share = float((ops.compams_dropout(torch.ones_like(x), 0.1, 12) == 0).float().mean())
    assert abs(share - R.threshold(0.1) / 65536) < 5 * math.sqrt(0.1 * 0.9 / 64000)
    empty = torch.empty(0, 10, device="cuda")
    assert ops.compams_dropout(empty, 0.5, 1).shape == (0, 10)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 63, 100, 513, 1000, 2048, 4099, 8193, 16390, 32003, 50257, 65537, 131073])
def test_cross_entropy(vocab, dtype):
    rng = np.random.default_rng(vocab)
    n, rows = 2, 9
    for pad, shift, target_type in ((0, 0, torch.int64), (vocab % 2 + 6, 1, torch.int32)):
        x, x64 = matrix(rng, n * rows, vocab, dtype, pad, shift, 3.0)
        t = torch.from_numpy(rng.integers(0, vocab, n * rows))
        t[1], t[n * rows - 1], t[3], t[4] = -100, -100, 0, vocab - 1
        scale = 2.0 ** 14 if dtype is F16 else 0.25
        dl, base = room(n * rows, vocab, dtype, pad, shift)
        got = ops.compams_cross_entropy(x, t.to(target_type).cuda(), n, grad_scale=scale, dlogits=dl)
        want, bound = R.cross_entropy(x64, t, n, -100, scale, dtype)
        for g, w, b, what in zip(got, want, bound, ("mean_loss", "losses", "dlogits")):
            R.close(g, w, b, what)
        untouched(base, shift, vocab)
        only = ops.compams_cross_entropy(x, t.to(target_type).cuda(), n, gradient=False)
        assert only[2] is None and torch.equal(only[0], got[0]) and torch.equal(only[1], got[1])


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [5, 777, 9000, 70000, 140000])
def test_cross_entropy_of_strange_rows(vocab, dtype):
    """Masked vocabulary, rows that a mask leaves empty, infinities, NaN, and targets that are none."""
    rng = np.random.default_rng(vocab + 1)
    n, rows = 2, 8
    v = torch.from_numpy(rng.standard_normal((n * rows, vocab)) * 2).to(dtype)
    lowest = torch.finfo(dtype).min
    t = torch.from_numpy(rng.integers(0, vocab, n * rows))
    t[0] = 1
    v[0, 2:] = -math.inf                 # two entries left
    v[1, :] = lowest                     # all masked by the lowest value: uniform
    v[2, :] = lowest
    v[2, t[2]] = torch.finfo(dtype).max  # as far apart as the type allows
    v[3, t[3]] = -math.inf               # the target itself masked: an infinite loss
    v[4, :] = -math.inf                  # nothing left: none
    v[5, vocab // 2] = math.inf
    v[6, vocab - 1] = math.nan
    t[7], t[8] = -1, vocab               # no column
    t[9], v[9, :] = -100, math.nan       # ignored, whatever stands there
    t[10], v[10, :] = -100, -math.inf
    v[11, :] = lowest
    v[11, t[11]] = 0.0
    got = ops.compams_cross_entropy(v.cuda(), t.cuda(), n, grad_scale=512.0)
    want, bound = R.cross_entropy(v.double(), t, n, -100, 512.0, dtype)
    for w in want[1:]:                   # a row of minus infinities has no softmax
        w[4] = math.nan
    want[0][0] = math.nan
    for g, w, b, what in zip(got, want, bound, ("mean_loss", "losses", "dlogits")):
        R.close(g, w, b, what)
    assert bool(torch.isinf(got[1][3])) and bool(torch.isnan(got[1][4:9]).all()) and float(got[1][9]) == 0
    assert bool((got[2][9:11] == 0).all()) and bool(torch.isnan(got[2][7:9]).all())


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [40, 1500, 20000, 140000])
def test_cross_entropy_far_from_zero(vocab, dtype):
    """Rows whose logits are a few steps of the type apart, at every magnitude that the type has."""
    tops = [1e3, 3e4, -6e4] if dtype is F16 else [1e3, 1e6, 1e8, 1e9, 4e9, 1e10, 3e12, 1e20, 1e30, 3e38, -1e6, -1e9, -1e10, -1e25, -3e38]
    rng = np.random.default_rng(vocab)
    rows = len(tops)
    v = torch.tensor(tops, dtype=torch.float64)[:, None].expand(rows, vocab).to(dtype).clone()
    for _ in range(8):
        down = torch.from_numpy(rng.random((rows, vocab)) < 0.5)
        v = torch.where(down, torch.nextafter(v, torch.tensor(-math.inf, dtype=dtype)), v)
    v = torch.where(torch.isfinite(v), v, torch.finfo(dtype).min)
    t = torch.from_numpy(rng.integers(0, vocab, rows))
    got = ops.compams_cross_entropy(v.cuda(), t.cuda(), 1, grad_scale=64.0)
    want, bound = R.cross_entropy(v.double(), t, 1, -100, 64.0, dtype)
    for g, w, b, what in zip(got, want, bound, ("mean_loss", "losses", "dlogits")):
        R.close(g, w, b, what)


def test_workers_without_tokens():
    x = torch.randn(6, 40, device="cuda")
    t = torch.tensor([1, 2, 7, 7, 7, 3], device="cuda")
    mean, losses, d = ops.compams_cross_entropy(x, t, 3, ignore_index=7)
    assert float(mean[1]) == 0 and bool((losses[2:4] == 0).all()) and bool((d[2:4] == 0).all())
    want, bound = R.cross_entropy(x.cpu().double(), t.cpu(), 3, 7, 1.0, F32)
    R.close(mean, want[0], bound[0], "mean_loss")
    R.close(d, want[2], bound[2], "dlogits")
    # no rows at all
    mean, losses, d = ops.compams_cross_entropy(torch.empty(0, 40, device="cuda"), t[:0], 3)
    assert torch.equal(mean.cpu(), torch.zeros(3)) and losses.numel() == 0 and d.shape == (0, 40)
    many = ops.compams_cross_entropy(torch.randn(5000, 24, device="cuda"), torch.zeros(5000, dtype=torch.int64, device="cuda"), 1)
    assert bool(torch.isfinite(many[0]).all())


def test_no_rows():
    e = torch.empty(0, 100, device="cuda")
    z = torch.empty(0, device="cuda")
    gamma = torch.ones(100, device="cuda")
    assert ops.compams_layer_norm_forward(e, gamma, gamma)[0].shape == (0, 100)
    for n in (1, 4):
        dg = torch.full((n, 100), 5.0, device="cuda")
        out = ops.compams_layer_norm_backward(e, e, z, z, gamma, n, dgamma=dg)
        assert bool((dg == 0).all()) and bool((out[2] == 0).all())
        dg.fill_(5.0)
        ops.compams_layer_norm_backward(e, e, z, z, gamma, n, dgamma=dg, dbeta=dg.clone(), accumulate=True)
        assert bool((dg == 5.0).all())


def differences(f, direction, at, step=1e-5):
    return (f(at + step * direction) - f(at - step * direction)) / (2 * step)


@pytest.mark.parametrize("cols", [40, 768, 2500])
def test_gradients_against_differences(cols):
    """Central differences, in 64 bits, of the whole path from the branch to a loss: cross-entropy of the joined and
    normed rows, in random directions of every input and weight."""
    rng = np.random.default_rng(cols)
    n, rows, p, seed, offset = 2, 6, 0.25, 21, 22
    make = lambda *s: torch.from_numpy(rng.standard_normal(s)).float().double()  # noqa: E731
    inputs = {"x": make(n * rows, cols), "residual": make(n * rows, cols), "bias": make(cols), "gamma": make(cols), "beta": make(cols)}
    t = torch.from_numpy(rng.integers(0, cols, n * rows))
    t[2] = -100
    keep = R.kept(n * rows, cols, p, seed, offset)

    def losses(v):
        h = v["residual"] + torch.where(keep, (v["x"] + v["bias"]) * R.factor(p), 0.0)
        y = R.norm_forward(h, v["gamma"], v["beta"], EPS, F32)[0][0]
        return R.cross_entropy(y, t, n, -100, 1.0, F32)[0][0]

    dev = {k: v.float().cuda() for k, v in inputs.items()}
    h, y, mean, rstd = ops.compams_dropout_add_norm_forward(dev["x"], dev["residual"], dev["gamma"], dev["beta"], p, seed, offset,
                                                            EPS, bias=dev["bias"])
    loss, _, dy = ops.compams_cross_entropy(y, t.cuda(), n)
    got = ops.compams_dropout_add_norm_backward(dy, None, h, mean, rstd, dev["gamma"], p, seed, offset, n)
    grad = dict(zip(("x", "residual", "gamma", "beta", "bias"), (g.cpu().double() for g in got)))
    assert torch.allclose(loss.cpu().double(), losses(inputs), rtol=1e-5)
    for name, g in grad.items():
        for _ in range(3):
            d = make(*inputs[name].shape)
            want = differences(lambda v: losses(dict(inputs, **{name: v})), d, inputs[name])    # one for each worker
            have = (g * d).sum(1) if g.shape[0] == n and name in ("gamma", "beta", "bias") else \
                (g * d).reshape(n, rows * cols).sum(1)
            # the differences: step^2 times a third derivative of order 1; the gradient: 32-bit rounding of its terms
            size = (g * d).abs().reshape(n, -1).sum(1)
            assert bool(((want - have).abs() <= 1e-6 * size + 1e-7).all()), (name, want, have)


def test_rows_beyond_32_bits():
    """Three rows 2^31 elements apart: the last one starts 2^32 elements into its buffer."""
    far, cols = 1 << 31, 1500
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 60 GB")
    rng = np.random.default_rng(4)
    base = torch.empty(2 * far + cols, dtype=BF16, device="cuda")
    x = torch.as_strided(base, (3, cols), (far, 1))
    v = torch.from_numpy(rng.standard_normal((3, cols))).to(BF16)
    x.copy_(v.cuda())
    near = v.cuda()
    base2 = torch.empty(2 * far + cols, dtype=BF16, device="cuda")
    out = torch.as_strided(base2, (3, cols), (far, 1))
    gamma, beta = vector(rng, cols, 1.0)[0], vector(rng, cols)[0]
    t = torch.tensor([5, 6, 7], device="cuda")
    ops.compams_layer_norm_forward(x, gamma, beta, y=out)
    y, mean, rstd = ops.compams_layer_norm_forward(near, gamma, beta)
    assert torch.equal(out, y)
    ops.compams_layer_norm_backward(x, x, mean, rstd, gamma, dx=out)
    assert torch.equal(out, ops.compams_layer_norm_backward(near, near, mean, rstd, gamma)[0])
    ops.compams_dropout(x, 0.3, 1, residual=x, y=out)
    assert torch.equal(out, ops.compams_dropout(near, 0.3, 1, residual=near))
    ops.compams_cross_entropy(x, t, dlogits=out)
    assert torch.equal(out, ops.compams_cross_entropy(near, t)[2])


def test_other_streams_and_graphs():
    """Work goes to the current stream; a recorded step draws new masks on every replay through the device's counter."""
    rng = np.random.default_rng(6)
    n, rows, cols, p, seed = 2, 40, 768, 0.2, 3
    x = matrix(rng, n * rows, cols, F32)[0]
    gamma, beta = vector(rng, cols, 1.0)[0], vector(rng, cols)[0]
    t = torch.from_numpy(rng.integers(0, cols, n * rows)).cuda()
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def once(step=None, offset=0):
        h, y, mean, rstd = ops.compams_dropout_add_norm_forward(x, x, gamma, beta, p, seed, offset, step=step)
        loss, losses, dy = ops.compams_cross_entropy(y, t, n)
        back = ops.compams_dropout_add_norm_backward(dy, None, h, mean, rstd, gamma, p, seed, offset, n, step=step)
        return (h, y, loss, losses, ops.compams_dropout(x, p, seed, offset, step=step)) + back

    want = [[v.clone() for v in once(offset=k)] for k in range(4)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = once(offset=2)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[2]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        once(step)
    side.synchronize()
    with torch.cuda.graph(graph):
        out = once(step)
    for k in (1, 3, 0, 2):
        step.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[k])), k
        torch.empty(1 << 20, device="cuda").fill_(float(k)).sum().item()     # the program's own work in between


def test_refusals():
    x = torch.randn(6, 32, device="cuda")
    g = torch.ones(32, device="cuda")
    s = torch.ones(6, device="cuda")
    t = torch.zeros(6, dtype=torch.int64, device="cuda")
    for call in (lambda: ops.compams_layer_norm_forward(x.double(), g, g),
                 lambda: ops.compams_layer_norm_forward(x.t(), torch.ones(6, device="cuda"), None),
                 lambda: ops.compams_layer_norm_forward(x, g[:31], g),
                 lambda: ops.compams_layer_norm_forward(x, g.half(), g),
                 lambda: ops.compams_layer_norm_forward(x, g.cpu(), g),
                 lambda: ops.compams_layer_norm_forward(x.cpu(), None, None),
                 lambda: ops.compams_layer_norm_forward(x[0], g, g),
                 lambda: ops.compams_layer_norm_forward(x, g, g, y=x[:, :16]),
                 lambda: ops.compams_layer_norm_forward(x.half(), g, g, y=x.bfloat16()),
                 lambda: ops.compams_layer_norm_forward(x.half(), g, g, dtype=F32),
                 lambda: ops.compams_layer_norm_forward(x, g, g, -1.0),
                 lambda: ops.compams_layer_norm_forward(x, g, g, math.nan),
                 lambda: ops.compams_layer_norm_forward(x[:1].expand(6, 32), g, g),
                 lambda: ops.compams_layer_norm_backward(x, x, s, s, g, 4),
                 lambda: ops.compams_layer_norm_backward(x, x, s, s, g, 0),
                 lambda: ops.compams_layer_norm_backward(x, x, s[:5], s, g),
                 lambda: ops.compams_layer_norm_backward(x, x, s, s, g, accumulate=True),
                 lambda: ops.compams_layer_norm_backward(x, x, s, s, g, 2, dgamma=torch.zeros(2, 31, device="cuda")),
                 lambda: ops.compams_layer_norm_backward(x, x.half(), s, s, g),
                 lambda: ops.compams_dropout(x, 1.5, 1), lambda: ops.compams_dropout(x, -0.1, 1),
                 lambda: ops.compams_dropout(x, math.nan, 1), lambda: ops.compams_dropout(x.half(), 0.1, 1, dtype=BF16),
                 lambda: ops.compams_dropout(x, 0.1, 1, residual=x[:3]),
                 lambda: ops.compams_dropout(x, 0.1, 1, step=t[:2]),
                 lambda: ops.compams_dropout(x, 0.1, 1, step=s[:1]),
                 lambda: ops.compams_dropout_add_norm_forward(x, x.half(), g, g, 0.1, 1),
                 lambda: ops.compams_dropout_add_norm_forward(x, x, g, g, 2.0, 1),
                 lambda: ops.compams_cross_entropy(x, t[:5]), lambda: ops.compams_cross_entropy(x, s),
                 lambda: ops.compams_cross_entropy(x, t, 4), lambda: ops.compams_cross_entropy(x, t.cpu()),
                 lambda: ops.compams_cross_entropy(x, t, workspace=torch.empty(0, dtype=torch.uint8, device="cuda")),
                 lambda: ops.compams_cross_entropy(x, t, gradient=False, dlogits=x)):
        with pytest.raises((ValueError, B.CompamsError)):
            call()


@pytest.mark.parametrize("types", [(F16, F16), (BF16, F32)], ids=["f16", "bf16_f32"])
@pytest.mark.parametrize("cols", [68, 72, 173, 200, 300, 321, 330, 384, 385, 450, 512, 2304, 2500, 2900, 3008, 5400, 6144, 7169,
                                  10484, 16384, 20479, 20480])
def test_layer_norm_of_every_kind_of_team(cols, types):
    test_layer_norm(cols, types)


@pytest.mark.parametrize("types", [(F16, F16), (BF16, F32)], ids=["f16", "bf16_f32"])
@pytest.mark.parametrize("cols", [68, 173, 200, 300, 321, 330, 384, 450, 512, 1111, 1280, 1792, 2304, 2900, 7169, 16384, 20480])
def test_join_between_the_teams_widths(cols, types):
    test_join(cols, types)


@pytest.mark.parametrize("n,rows,cols", [(1, 513, 1111), (2, 600, 1280), (2, 512, 1600), (2, 513, 1792), (3, 128, 2500), (3, 129, 2500),
                                         (2, 40, 200), (2, 200, 68), (2, 70, 512), (2, 9, 8300), (2, 3, 4100), (1, 5, 9000)])
def test_sums_of_parts_of_every_size(n, rows, cols):
    test_sums_over_any_number_of_rows(n, rows, cols)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("vocab", [64, 65, 127, 129, 250, 260, 385, 500, 1030, 2047, 2050, 33000, 40007, 49160, 70001, 81930, 98304])
def test_cross_entropy_of_every_kind_of_team(vocab, dtype):
    test_cross_entropy(vocab, dtype)


@pytest.mark.parametrize("n,rows,vocab", [(2, 512, 90), (2, 513, 90), (1, 1100, 260), (3, 8200, 24), (9, 700, 130), (1, 530, 2200)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_cross_entropy_of_many_rows(n, rows, vocab, dtype):
    test_cross_entropy_of_many_shapes(n, rows, vocab, dtype)


@pytest.mark.parametrize("rows,vocab", [(4, 40), (32, 300), (3, 2000), (33, 40), (600, 24)])
def test_a_worker_on_its_own_has_the_same_loss(rows, vocab):
    """The bits of a worker's loss and gradient do not depend on how many workers stand beside it."""
    rng = np.random.default_rng(rows * vocab)
    n = 300 if rows <= 32 else 40
    x, _ = matrix(rng, n * rows, vocab, BF16, 0, 0, 2.0)
    t = torch.from_numpy(rng.integers(0, vocab, n * rows)).cuda()
    t[::7] = -100
    beside = ops.compams_cross_entropy(x, t, n)
    for w in (0, n - 1):
        part = slice(w * rows, (w + 1) * rows)
        alone = ops.compams_cross_entropy(x[part], t[part], 1)
        assert torch.equal(alone[0][0], beside[0][w])
        assert torch.equal(alone[1], beside[1][part]) and torch.equal(alone[2], beside[2][part])
