"""The norm of every worker's gradient and its bound, on the GPU against the formulas in 64 bits."""
import math

import pytest
import torch

from operator_reference import U, UNIT, LEAST, close
from paper_2205_05632_amd import binding as B
from paper_2205_05632_amd import operators as ops

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def reference(tensors, max_norm, scale):
    """norms, factors and each tensor times its factor, on the host.  (max_norm and scale are fp32 arguments.)"""
    max_norm, scale = (float(torch.tensor(v, dtype=F32)) for v in (max_norm, scale))
    wide = [t.cpu().double() for t in tensors]
    squares = sum(t.square().sum(1) for t in wide)
    norms = scale * squares.sqrt()
    factors = torch.where(norms > max_norm, scale * (max_norm / norms), torch.full_like(norms, scale))
    factors = torch.where(torch.isfinite(squares), factors, 0.0)
    return [torch.where(factors[:, None] == 0, 0.0, t * factors[:, None]) for t in wide], norms, factors


def check(got, want, dtypes):
    out, norms, factors = got
    # the norm is rounded once (its sum has 53 bits), the factor too, an entry once after the factor
    close(norms, want[1], 1.01 * U * want[1].abs() + 2.0 ** -149, "norms")
    close(factors, want[2], 1.01 * U * want[2].abs() + 2.0 ** -149, "factors")
    for o, w, dtype in zip(out, want[0], dtypes):
        close(o, w, (UNIT[dtype] + 2.1 * U) * w.abs() + LEAST[dtype], "out")


COUNTS = [1, 2, 7, 8, 9, 255, 2048, 2049, 8191, 8192, 8193, 50000, 300001]


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("count", COUNTS)
def test_one_tensor(count, dtype):
    """Rows that start anywhere, some of them above the bound and some below; what lies between them is left alone."""
    g = torch.Generator(device="cuda").manual_seed(count)
    n = 3
    base = torch.full((n, count + 5), math.nan, dtype=dtype, device="cuda")
    x = base[:, 1:1 + count]
    x.copy_((torch.randn((n, count), generator=g, device="cuda") * torch.tensor([[0.01], [1.0], [3.0]], device="cuda")).to(dtype))
    max_norm = 0.7 * math.sqrt(count)
    for out_type in {dtype, F32}:
        room = torch.full((n, count + 3), 7.0, dtype=out_type, device="cuda")
        got = ops.compams_clip_gradients(x, max_norm, n, scale=0.5, out=room[:, 2:2 + count])
        check(([got[0]], *got[1:]), reference([x], max_norm, 0.5), [out_type])
        assert bool((room[:, :2] == 7).all()) and bool((room[:, 2 + count:] == 7).all())
    want = reference([x], max_norm, 1.0)
    got = ops.compams_clip_gradients(x, max_norm, n)
    assert got[0] is x
    check(([x], *got[1:]), want, [dtype])
    assert bool(torch.isnan(base[:, 0]).all()) and bool(torch.isnan(base[:, 1 + count:]).all())


def test_many_tensors_of_mixed_types():
    """More tensors than a launch takes, empty ones among them, into places of a gradient buffer's rows."""
    g = torch.Generator(device="cuda").manual_seed(9)
    n, types = 2, [F32, F16, BF16]
    sizes = [(i * 37) % 501 * (1 if i % 5 else 40) for i in range(150)]
    tensors = [(torch.randn((n, s), generator=g, device="cuda") * (0.5 + i % 7)).to(types[i % 3]) for i, s in enumerate(sizes)]
    rows = torch.full((n, sum(sizes) + 4), 7.0, device="cuda")
    out = list(rows[:, 1:1 + sum(sizes)].split(sizes, 1))
    want = reference(tensors, 12.5, 2.0 ** -3)
    got = ops.compams_clip_gradients(tensors, 12.5, n, scale=2.0 ** -3, out=out)
    check(got, want, [F32] * len(sizes))
    assert bool((rows[:, 0] == 7).all()) and bool((rows[:, -3:] == 7).all())
    again = [t.clone() for t in got[0]]
    ops.compams_clip_gradients(tensors, 12.5, n, scale=2.0 ** -3, out=out)
    assert all(torch.equal(a, b) for a, b in zip(again, out))


@pytest.mark.parametrize("count", [5, 3000, 20000])
def test_gradients_that_are_not_finite(count):
    """Such a worker's norm says so and its gradient becomes 0; the others are not touched by it."""
    x = torch.randn((5, count), generator=torch.Generator().manual_seed(1)).cuda()
    x[1, count - 1], x[2, 0], x[4, 1] = math.nan, math.inf, -math.inf
    x[4, 2] = math.nan
    want = reference([x], 1.0, 1.0)
    out, norms, factors = ops.compams_clip_gradients(x, 1.0, 5)
    check(([out], norms, factors), want, [F32])
    assert not bool(out[1].any()) and not bool(out[2].any()) and not bool(out[4].any()) and bool(torch.isfinite(out).all())
    assert math.isinf(float(norms[2])) and math.isnan(float(norms[1])) and math.isnan(float(norms[4]))


@pytest.mark.parametrize("size", [1e-44, 1e-30, 1e-20, 1e15, 1e30, 3e38])
def test_gradients_of_any_size(size):
    """Squares that fp32 has no room for."""
    x = torch.full((2, 300), size, device="cuda")
    x[1, 7:] = 0
    want = reference([x], 1.0, 1.0)
    # (the norm of 300 entries of 3e38 is beyond fp32's range: infinite as it is rounded, the factor as it should be)
    norms32 = want[1].float().double()
    out, norms, factors = ops.compams_clip_gradients(x, 1.0, 2)
    close(norms, norms32, 2.02 * U * norms32.abs().nan_to_num(posinf=0.0) + 2.0 ** -148, "norms")
    close(factors, want[2], 1.01 * U * want[2] + 2.0 ** -149, "factors")
    close(out, want[0][0], 2.2 * U * want[0][0].abs() + 3.4e38 * 2.0 ** -149, "out")


def test_bounds_of_zero_and_infinity_and_gradients_of_zero():
    x = torch.randn((3, 100), generator=torch.Generator().manual_seed(2)).cuda()
    x[1] = 0.0
    before = x.clone()
    _, norms, factors = ops.compams_clip_gradients(x, math.inf, 3)
    assert torch.equal(x, before) and bool((factors == 1).all()) and float(norms[1]) == 0.0
    out, _, factors = ops.compams_clip_gradients(x, 0.0, 3, out=torch.empty_like(x))
    assert not bool(out.any()) and factors.tolist() == [0.0, 1.0, 0.0]


def test_a_worker_alone_is_the_same_bits():
    x = torch.randn((7, 30011), generator=torch.Generator().manual_seed(3)).cuda()
    out, norms, factors = ops.compams_clip_gradients(x, 2.0, 7, out=torch.empty_like(x))
    one = ops.compams_clip_gradients(x[4:5], 2.0, 1, out=torch.empty_like(x[4:5]))
    assert torch.equal(one[0], out[4:5]) and torch.equal(one[1], norms[4:5]) and torch.equal(one[2], factors[4:5])


def test_captured_and_on_another_stream():
    """Into the rows that a step reads, and the step, recorded into a graph; replays against eager calls."""
    n, d = 3, 20000
    g = torch.Generator(device="cuda").manual_seed(5)
    src = [torch.randn((n, s), generator=g, device="cuda").half() for s in (15000, 5000)]
    rows = torch.zeros((n, B.padded_ld(d)), device="cuda")
    out, norms, factors = [rows[:, :15000], rows[:, 15000:20000]], torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    space = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    call = lambda: ops.compams_clip_gradients(src, 30.0, n, out=out, norms=norms, factors=factors, workspace=space)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(3):
        for t in src:
            t.copy_(torch.randn(t.shape, generator=g, device="cuda") * (0.1 + turn))
        call()
        eager = [rows.clone(), norms.clone(), factors.clone()]
        for t in (rows, norms, factors):
            t.fill_(3.0)
        rows[:, d:] = eager[0][:, d:]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, (rows, norms, factors)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,out_type", [(F32, F32), (BF16, F32), (F16, F16)])
def test_more_than_the_caches_hold(dtype, out_type):
    """Gradients of more than 192 MB, in three tensors that start anywhere."""
    g = torch.Generator(device="cuda").manual_seed(8)
    n, sizes = 2, [27_000_001, 4097, 25_000_000]
    base = torch.randn((n, sum(sizes) + 3), generator=g, device="cuda").to(dtype)
    tensors = [base[:, 1 + sum(sizes[:i]):1 + sum(sizes[:i + 1])] for i in range(3)]
    room = torch.full((n, sum(sizes) + 2), 7.0, dtype=out_type, device="cuda")
    out = list(room[:, 1:1 + sum(sizes)].split(sizes, 1))
    _, norms, factors = ops.compams_clip_gradients(tensors, 100.0, n, scale=0.5, out=out)
    want = base[:, 1:1 + sum(sizes)].double().square().sum(1).sqrt() * 0.5
    close(norms, want.cpu(), 1.01 * U * want.cpu(), "norms")
    factor = 0.5 * 100.0 / want
    close(factors, factor.cpu(), 1.01 * U * factor.cpu(), "factors")
    got, exact = room[:, 1:1 + sum(sizes)].double(), base[:, 1:1 + sum(sizes)].double() * factor[:, None]
    assert bool(((got - exact).abs() <= (UNIT[out_type] + 2.1 * U) * exact.abs() + LEAST[out_type]).all())
    assert bool((room[:, 0] == 7).all()) and bool((room[:, -1] == 7).all())
