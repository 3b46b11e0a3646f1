"""Forms of the operators' kernels that a size, a type or an absent argument picks: each against the formulas in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

import operator_reference as R
from paper_2205_05632_amd import binding as B
from paper_2205_05632_amd import operators as ops
from test_gpu_operators import BF16, EPS, F16, F32, IDS, TYPES, matrix, room, test_dropout as dropout_test, untouched, vector

pytestmark = pytest.mark.gpu


def norm_without(what, cols, types, rows=5):
    """A layer norm forward, through the C ABI, with the arguments in `what` left out."""
    dtype, stream = types
    rng = np.random.default_rng(cols + TYPES.index(types))
    x, x64 = matrix(rng, rows, cols, stream, 8, 0, 2.0)
    gamma, g64 = vector(rng, cols, 1.0)
    beta, b64 = vector(rng, cols)
    y, base = room(rows, cols, dtype, 8)
    mean, rstd = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
    given = {"gamma": gamma, "beta": beta, "mean": mean, "rstd": rstd}
    a = ops.compams_norm(n=1, rows=rows, cols=cols, type=ops._TYPE[dtype], stream_type=ops._TYPE[stream], eps=EPS, h=x.data_ptr(),
                         ld_h=cols + 8, y=y.data_ptr(), ld_y=cols + 8)
    for k, t in given.items():
        setattr(a, k, None if k in what else t.data_ptr())
    assert B.lib().compams_layer_norm_forward(ctypes.byref(a), torch.cuda.current_stream().cuda_stream) == 0
    g64 = torch.ones_like(g64) if "gamma" in what else g64
    b64 = torch.zeros_like(b64) if "beta" in what else b64
    want, bound = R.norm_forward(x64, g64, b64, EPS, dtype)
    R.close(y, want[0], bound[0], "y")
    untouched(base, 0, cols)
    for k, w, b in zip(("mean", "rstd"), want[1:], bound[1:]):
        if k in what:
            assert bool((given[k] == 7.0).all())
        else:
            R.close(given[k], w, b, k)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("what", [(), ("gamma",), ("beta",), ("gamma", "beta"), ("mean",), ("mean", "rstd")],
                         ids=lambda w: "without_" + "_".join(w) if w else "all")
@pytest.mark.parametrize("cols", [1600, 16392, 20008, 30008, 32760, 32768])
def test_wide_norms_of_whole_groups(cols, what, types):
    """Rows that a workgroup holds four groups a lane of, lanes idle or none, and the same rows in calls that leave something
    out, which another route takes."""
    norm_without(what, cols, types)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("cols", [768, 1600, 1792])
@pytest.mark.parametrize("what", ["bias", "residual", "gamma", "beta"])
def test_joins_without(what, cols, types):
    """Joins of whole groups that leave one argument out."""
    dtype, stream = types
    rng = np.random.default_rng(cols + TYPES.index(types))
    total, p, seed = 21, 0.2, 77
    x, x64 = matrix(rng, total, cols, dtype)
    res, r64 = matrix(rng, total, cols, stream, 0, 0, 2.0)
    (gamma, g64), (beta, b64), (bias, c64) = vector(rng, cols, 1.0), vector(rng, cols), vector(rng, cols)
    h = torch.empty(total, cols, dtype=stream, device="cuda")
    args = {"residual": res, "gamma": gamma, "beta": beta, "bias": bias}
    args[what] = None
    _, y, mean, rstd = ops.compams_dropout_add_norm_forward(x, args["residual"], args["gamma"], args["beta"], p, seed, bias=args["bias"],
                                                            h=h)
    one, zero = torch.ones_like(g64), torch.zeros_like(g64)
    g64, b64, c64 = (one if what == "gamma" else g64), (zero if what == "beta" else b64), (zero if what == "bias" else c64)
    r64 = torch.zeros_like(r64) if what == "residual" else r64
    branch = torch.where(R.kept(total, cols, p, seed, 0), (x64 + c64) * R.factor(p), torch.zeros_like(x64))
    h64 = r64 + branch
    R.close(h, h64, R.rounding(h64, stream) + 4.04 * R.U * (branch.abs() + h64.abs()), "h")
    want, bound = R.norm_forward(h64, g64, b64, EPS, dtype)
    for got, w, b, name in zip((y, mean, rstd), want, bound, ("y", "mean", "rstd")):
        R.close(got, w, b, name)


def counted_first(n, rows, vocab, dtype=BF16, targets=torch.int64):
    """Whether a call counts the workers' targets in a launch of its own, which leaves the counts at its workspace's start; its
    outputs are checked on the way."""
    g = torch.Generator(device="cuda").manual_seed(n + rows + vocab)
    x = torch.randn(n * rows, vocab, generator=g, device="cuda").to(dtype)
    t = torch.randint(0, vocab, (n * rows,), generator=g, device="cuda").to(targets)
    t[::3] = -100
    ws = torch.full((1 << 16,), 0x5A, dtype=torch.uint8, device="cuda")
    mean, losses, _ = ops.compams_cross_entropy(x, t, n, dlogits=x, workspace=ws)
    count = (t != -100).reshape(n, rows).sum(1)
    assert torch.allclose(mean.double() * count, losses.double().reshape(n, rows).sum(1), rtol=1e-5)
    head = ws[:4 * n].view(torch.int32)
    if bool((ws[:4 * n] == 0x5A).all()):
        return False
    assert torch.equal(head, count.int())
    return True


@pytest.mark.parametrize("n,rows,vocab,launch", [(1, 8000, 33000, True), (8, 1100, 8192, True), (1, 4100, 16500, True), (1, 2000, 8192, False),
                                                 (8, 500, 1000, False), (1, 1100, 260, True)])
def test_many_targets_are_counted_once(n, rows, vocab, launch):
    """Every row's team counts its worker's targets only where those are few, and not because the rows are long."""
    assert counted_first(n, rows, vocab) == launch


@pytest.mark.parametrize("n,rows,vocab", [(5000, 32, 100), (5000, 30, 24), (300, 32, 1000)])
@pytest.mark.parametrize("targets", [torch.int32, torch.int64], ids=["i32", "i64"])
def test_few_rows_of_many_workers_are_one_launch(n, rows, vocab, targets):
    """A workgroup that has all of a worker's rows counts them: no launch for that, however many workers there are."""
    assert not counted_first(n, rows, vocab, targets=targets)


@pytest.mark.parametrize("kinds", [(F32, F32), (F16, F16), (BF16, BF16), (F32, F16), (F32, BF16), (F16, F32), (BF16, F32)],
                         ids=lambda k: f"{k[0]}_{k[1]}".replace("torch.", ""))
@pytest.mark.parametrize("total,cols", [(37, 512), (9, 1000), (23, 1024), (37, 1536), (1, 2048), (11, 6000), (6, 16384)])
def test_dropout_of_rows_that_fill_wavefronts(total, cols, kinds):
    """Whole groups, 64 lanes side by side and more, rows that end within a workgroup's turn: alone and added to a stream."""
    dropout_test(total, cols, kinds)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,rows,vocab,pad", [(1100, 32, 1000, 0), (7, 2500, 1000, 0), (8, 4096, 600, 1), (3, 1800, 4096, 0), (2, 1100, 9000, 8),
                                              (2, 240, 50257, 0), (3, 90, 70001, 0), (2, 70, 140000, 0)])
def test_gradients_that_do_not_fit_the_cache(n, rows, vocab, pad, dtype):
    """Gradients of more than 32 MB are streamed past it: every kind of team, beside the logits and over them."""
    assert n * rows * vocab * 2 > 32 << 20
    rng = np.random.default_rng(vocab)
    g = torch.Generator(device="cuda").manual_seed(vocab + n)
    base = torch.randn(n * rows, vocab + pad, generator=g, device="cuda").mul_(2.5).to(dtype)
    x = base[:, :vocab]
    t = torch.from_numpy(rng.integers(0, vocab, n * rows)).cuda()
    t[::5] = -100
    dl, out = room(n * rows, vocab, dtype, pad)
    got = ops.compams_cross_entropy(x, t, n, grad_scale=64.0, dlogits=dl)
    want, bound = R.cross_entropy(x.double(), t, n, -100, 64.0, dtype)
    for a, w, b, what in zip(got, want, bound, ("mean_loss", "losses", "dlogits")):
        R.close(a, w.cpu(), b.cpu(), what)
    untouched(out, 0, vocab)
    over = ops.compams_cross_entropy(x, t, n, grad_scale=64.0, dlogits=x)
    assert over[2].data_ptr() == x.data_ptr() and all(torch.equal(a, b) for a, b in zip(over, got))
