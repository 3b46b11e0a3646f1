"""Calls of the C ABI that ask for some of an operator's outputs, on the GPU against the calls that ask for all."""
import ctypes
import math

import pytest
import torch

from paper_2205_05632_amd import binding as B
from paper_2205_05632_amd import operators as ops

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def call(name, a):
    """The call with a workspace of just the size that it asks for."""
    need = getattr(B.lib(), name.replace("_gradients", "").replace("_cross_entropy", "_loss") + "_workspace_size")(ctypes.byref(a))
    room = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = room.data_ptr(), need
    B._check(B._on_stream(torch.device("cuda", 0), getattr(B.lib(), name), ctypes.byref(a)), name)
    return room


def launches(run):
    """Kernels that a call enqueues."""
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        run()
    count, hip = ctypes.c_size_t(), ctypes.CDLL("libamdhip64.so")
    assert hip.hipGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(count)) == 0
    return count.value


def clip(tensors, n, norms, factors, to=None):
    kind = {F32: ops.F32, F16: ops.F16, BF16: ops.BF16}
    table = (ops.compams_clip_tensor * len(tensors))()
    for i, (row, t) in enumerate(zip(table, tensors)):
        o = to.get(i) if to else None
        for k, v in {"from": t.data_ptr(), "ld_from": t.stride(0), "to": None if o is None else o.data_ptr(),
                     "ld_to": 0 if o is None else o.stride(0), "count": t.shape[1], "from_type": kind[t.dtype],
                     "to_type": kind[t.dtype]}.items():
            setattr(row, k, v)
    a = ops.compams_clip(n=n, tensors=len(tensors), tensor=ctypes.addressof(table), max_norm=3.0, scale=0.5,
                         norms=norms.data_ptr() if norms is not None else None, factors=factors.data_ptr() if factors is not None else None)
    a.table = table
    return a


@pytest.mark.parametrize("n,sizes", [(1, [1]), (3, [100, 5000]), (2, [0, 30000]), (4, [7] * 150), (2, [27_000_001])])
def test_norms_alone(n, sizes):
    """Nothing is scaled: the norms' pass and one launch for what follows from it, however large the gradients are."""
    g = torch.Generator(device="cuda").manual_seed(n)
    tensors = [torch.randn((n, s), generator=g, device="cuda").to((F32, F16, BF16)[i % 3]) for i, s in enumerate(sizes)]
    before = [t.clone() for t in tensors]
    _, norms, factors = ops.compams_clip_gradients(tensors, 3.0, n, scale=0.5, out=[torch.empty_like(t) for t in tensors])
    got, f = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    call("compams_clip_gradients", clip(tensors, n, got, f))
    assert torch.equal(got, norms) and torch.equal(f, factors) and all(torch.equal(a, b) for a, b in zip(tensors, before))
    got.fill_(7.0)
    call("compams_clip_gradients", clip(tensors, n, got, None))
    assert torch.equal(got, norms)
    a = clip(tensors, n, got, f)
    room = call("compams_clip_gradients", a)
    passes = -(-sum(s > 0 for s in sizes) // 64)
    assert launches(lambda: B._on_stream(torch.device("cuda", 0), B.lib().compams_clip_gradients, ctypes.byref(a))) == passes + 1
    del room


@pytest.mark.parametrize("size", [3000, 27_000_001])
def test_norms_of_all_and_some_scaled(size):
    """The first tensor is only read, the second is scaled."""
    g = torch.Generator(device="cuda").manual_seed(size)
    tensors = [torch.randn((2, s), generator=g, device="cuda") for s in (size, size // 2)]
    out, norms, factors = ops.compams_clip_gradients(tensors, 3.0, 2, scale=0.5, out=[torch.empty_like(t) for t in tensors])
    second, got, f = torch.empty_like(tensors[1]), torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    call("compams_clip_gradients", clip(tensors, 2, got, f, {1: second}))
    assert torch.equal(got, norms) and torch.equal(f, factors) and torch.equal(second, out[1])


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,rows,cols,vocab", [(1, 1, 8, 3), (3, 40, 33, 130), (2, 200, 64, 5000), (2, 9000, 16, 4100)])
def test_gradients_of_the_output_layer_alone(n, rows, cols, vocab, dtype):
    """dx without dweight (a layer that is not trained), dweight without dx, one gradient and no loss, losses without their mean."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn((n * rows, cols), generator=g, device="cuda").to(dtype)
    w = (torch.randn((vocab, cols), generator=g, device="cuda") / math.sqrt(cols)).to(dtype)
    t = torch.randint(0, vocab, (n * rows,), generator=g, device="cuda")
    t[::7] = -100
    names = ("mean_loss", "losses", "dx", "dweight")
    all_of_it = dict(zip(names, ops.compams_linear_cross_entropy(x, w, t, n, -100, 8.0)))
    for some in (("dx",), ("dweight",), ("losses", "dx"), ("mean_loss", "dweight"), ("losses",), ("mean_loss",), ("losses", "dx", "dweight")):
        out = {k: torch.full_like(all_of_it[k], 7.0) for k in some}
        a = ops.compams_linear_loss(n=n, rows=rows, cols=cols, vocab=vocab, type={F32: ops.F32, F16: ops.F16, BF16: ops.BF16}[dtype],
                                    target_type=ops.I64, x=x.data_ptr(), ld_x=cols, weight=w.data_ptr(), ld_weight=cols, targets=t.data_ptr(),
                                    ignore_index=-100, grad_scale=8.0, ld_dx=cols, ld_dweight=cols, stride_dweight=vocab * cols,
                                    **{k: v.data_ptr() for k, v in out.items()})
        call("compams_linear_cross_entropy", a)
        for k, v in out.items():
            assert torch.equal(v, all_of_it[k]), (some, k)    # (no sum's order goes by what else is asked for)
