"""Host-only checks of the boundary of the operators with products and of the gradient's bound: the binding's structures and what
the entry points refuse before anything is enqueued (no GPU needed)."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2205_05632_amd import binding as B
from paper_2205_05632_amd import operators as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ["gated", "projections", "linear_loss", "clip_tensor", "clip"]


@pytest.mark.parametrize("name", NAMES)
def test_structures_match_the_header(tmp_path, name):
    struct = getattr(ops, "compams_" + name)
    fields = [f[0] for f in struct._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "compams.h"\nint main(void){\n'
                   + f'printf("%zu\\n", sizeof(compams_{name}));\n'
                   + "".join(f'printf("%zu\\n", offsetof(compams_{name}, {f}));\n' for f in fields) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert out[0] == ctypes.sizeof(struct)
    assert out[1:] == [getattr(struct, f).offset for f in fields]


@pytest.mark.parametrize("name", NAMES)
def test_packed_arguments_have_the_structures_layout(name):
    packer, struct = getattr(ops, "_" + name.upper()), getattr(ops, "compams_" + name)
    assert packer.size == ctypes.sizeof(struct)
    values = [i + 1.5 if kind is ctypes.c_float else i + 1 for i, (_, kind) in enumerate(struct._fields_)]
    got = struct.from_buffer_copy(packer.pack(*values))
    assert [getattr(got, f) for f, _ in struct._fields_] == values


FAKE, MORE, LAST = 0x1000, 0x100000, 0x200000    # never dereferenced: validation fails first


def gated(**kw):
    a = ops.compams_gated(n=2, rows=300, cols=16, hidden=8, type=ops.F32, activation=0, x=FAKE, ld_x=16, gate_weight=FAKE, ld_gate_weight=16,
                          up_weight=FAKE, ld_up_weight=16, m=FAKE, ld_m=8, gate=MORE, ld_gate=8, up=LAST, ld_up=8, dm=FAKE, ld_dm=8,
                          dgate=MORE, ld_dgate=8, dup=LAST, ld_dup=8)
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


BOTH = [(dict(n=0), -1), (dict(n=65536), -1), (dict(rows=-1), -1), (dict(rows=1 << 31), -1), (dict(n=65535, rows=65535), -1), (dict(hidden=0), -1),
        (dict(hidden=-1), -1), (dict(hidden=(1 << 20) + 1), -1), (dict(type=3), -1), (dict(type=-1), -1), (dict(activation=5), -1),
        (dict(activation=-1), -1), (dict(gate=FAKE + 2), -2), (dict(up=FAKE + 1), -2), (dict(ld_gate=7), -1), (dict(ld_up=7), -1)]


@pytest.mark.parametrize("kw,code", BOTH + [
    (dict(cols=0), -1), (dict(cols=(1 << 20) + 1), -1), (dict(x=None), -1), (dict(gate_weight=None), -1), (dict(up_weight=None), -1), (dict(m=None), -1),
    (dict(ld_x=15), -1), (dict(ld_gate_weight=15), -1), (dict(ld_up_weight=1), -1), (dict(ld_m=7), -1), (dict(x=FAKE + 2), -2),
    (dict(gate_weight=FAKE + 1), -2), (dict(up_weight=FAKE + 3), -2), (dict(m=FAKE + 2), -2), (dict(gate_bias=FAKE + 2), -2), (dict(up_bias=FAKE + 1), -2),
    (dict(x=FAKE + 4), -1), (dict(x=FAKE + 4, workspace=FAKE, workspace_bytes=100), -3),
    (dict(x=FAKE + 4, workspace=FAKE + 16, workspace_bytes=4096), -2), (dict(cols=15, ld_x=17), -1), (dict(ld_up_weight=17), -1), (dict(rows=0), 0),
    (dict(gate=FAKE), -1), (dict(up=FAKE), -1), (dict(gate=LAST), -1),
])
def test_gated_forward_refuses(kw, code):
    assert B.lib().compams_gated_forward(gated(**kw), None) == code


@pytest.mark.parametrize("kw,code", BOTH + [
    (dict(dgate=LAST), -1), (dict(dgate_bias=FAKE, ld_dgate_bias=8, dup_bias=FAKE, ld_dup_bias=8), -1), (dict(dm=None), -1), (dict(gate=None), -1), (dict(up=None), -1), (dict(dgate=None), -1), (dict(dup=None), -1), (dict(ld_dm=7), -1),
    (dict(ld_dgate=7), -1), (dict(ld_dup=7), -1), (dict(dm=FAKE + 2), -2), (dict(dgate=FAKE + 2), -2), (dict(dup=FAKE + 2), -2), (dict(accumulate=2), -1),
    (dict(dgate_bias=FAKE, ld_dgate_bias=7), -1), (dict(dup_bias=FAKE + 2, ld_dup_bias=8), -2),
    (dict(rows=100000, dgate_bias=FAKE, ld_dgate_bias=8), -1),
    (dict(rows=100000, dgate_bias=FAKE, ld_dgate_bias=8, workspace=FAKE, workspace_bytes=64), -3),
    (dict(rows=100000, dgate_bias=FAKE, ld_dgate_bias=8, workspace=FAKE + 8, workspace_bytes=1 << 30), -2), (dict(rows=0), 0),
])
def test_gated_backward_refuses(kw, code):
    assert B.lib().compams_gated_backward(gated(**kw), None) == code


def projections(**kw):
    a = ops.compams_projections(n=2, rows=3, cols=16, hidden=8, type=ops.F32, dgate=FAKE, ld_dgate=8, dup=FAKE, ld_dup=8, x=FAKE, ld_x=16,
                                gate_weight=FAKE, ld_gate_weight=16, up_weight=FAKE, ld_up_weight=16, dx=FAKE, ld_dx=16,
                                dgate_weight=FAKE, ld_dgate_weight=16, stride_dgate_weight=128, dup_weight=MORE, ld_dup_weight=16,
                                stride_dup_weight=128)
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), -1), (dict(rows=-1), -1), (dict(cols=0), -1), (dict(hidden=0), -1), (dict(cols=(1 << 20) + 1), -1), (dict(hidden=(1 << 20) + 1), -1),
    (dict(type=4), -1), (dict(dgate=None), -1), (dict(dup=None), -1), (dict(x=None), -1), (dict(gate_weight=None), -1), (dict(up_weight=None), -1),
    (dict(dx=None, dgate_weight=None, dup_weight=None), -1), (dict(dup_weight=FAKE), -1), (dict(ld_dgate=7), -1), (dict(ld_dup=7), -1), (dict(ld_x=15), -1), (dict(ld_dx=15), -1),
    (dict(ld_gate_weight=15), -1), (dict(ld_dgate_weight=15), -1), (dict(stride_dup_weight=15), -1), (dict(stride_dup_weight=-1), -1),
    (dict(dgate=FAKE + 2), -2), (dict(x=FAKE + 1), -2), (dict(dx=FAKE + 2), -2), (dict(up_weight=FAKE + 2), -2), (dict(dgate_weight=FAKE + 2), -2),
    (dict(accumulate=-1), -1), (dict(x=FAKE + 4), -1), (dict(x=FAKE + 4, workspace=FAKE, workspace_bytes=64), -3), (dict(n=65535, rows=1, hidden=1 << 20, cols=1 << 20), -1),
])
def test_projections_refuse(kw, code):
    assert B.lib().compams_projections_backward(projections(**kw), None) == code


def linear_loss(**kw):
    a = ops.compams_linear_loss(n=2, rows=3, cols=16, vocab=8, type=ops.F32, target_type=ops.I64, x=FAKE, ld_x=16, weight=FAKE, ld_weight=16,
                                targets=FAKE, grad_scale=1.0, mean_loss=FAKE, losses=FAKE, dx=FAKE, ld_dx=16, dweight=FAKE, ld_dweight=16,
                                stride_dweight=128, workspace=FAKE, workspace_bytes=1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), -1), (dict(rows=-1), -1), (dict(cols=0), -1), (dict(cols=(1 << 20) + 1), -1), (dict(vocab=0), -1), (dict(vocab=1 << 31), -1),
    (dict(type=ops.I32), -1), (dict(target_type=ops.F32), -1), (dict(x=None), -1), (dict(weight=None), -1), (dict(targets=None), -1), (dict(ld_x=15), -1),
    (dict(ld_weight=15), -1), (dict(ld_dx=15), -1), (dict(ld_dweight=15), -1), (dict(stride_dweight=15), -1), (dict(accumulate=2), -1),
    (dict(workspace=None), -1), (dict(workspace=FAKE + 16), -2), (dict(workspace_bytes=64), -3), (dict(x=FAKE + 2), -2), (dict(weight=FAKE + 2), -2),
    (dict(dx=FAKE + 2), -2), (dict(dweight=FAKE + 2), -2), (dict(losses=FAKE + 2), -2), (dict(mean_loss=FAKE + 1), -2), (dict(targets=FAKE + 4), -2),
    (dict(mean_loss=None, losses=None, dx=None, dweight=None), -1),
])
def test_linear_cross_entropy_refuses(kw, code):
    assert B.lib().compams_linear_cross_entropy(linear_loss(**kw), None) == code


def clip(entries=({},), **kw):
    table = (ops.compams_clip_tensor * max(1, len(entries)))()
    for t, more in zip(table, entries):
        for k, v in dict({"from": FAKE, "ld_from": 8, "to": FAKE, "ld_to": 8, "count": 8, "from_type": ops.F32, "to_type": ops.F32}, **more).items():
            setattr(t, k, v)
    a = ops.compams_clip(n=2, tensors=len(entries), tensor=ctypes.addressof(table), max_norm=1.0, scale=1.0, norms=FAKE, factors=FAKE,
                         workspace=FAKE, workspace_bytes=1 << 20)
    a.table = table
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("tensor,kw,code", [
    ({}, dict(n=0), -1), ({}, dict(n=65536), -1), ({}, dict(tensors=-1), -1), ({}, dict(tensor=None), -1), ({}, dict(max_norm=-1.0), -1),
    ({}, dict(max_norm=math.nan), -1), ({}, dict(scale=0.0), -1), ({}, dict(scale=-1.0), -1), ({}, dict(scale=math.inf), -1), ({}, dict(scale=math.nan), -1),
    ({}, dict(workspace=None), -1), ({}, dict(workspace=FAKE + 64), -2), ({}, dict(workspace_bytes=255), -3), ({}, dict(norms=FAKE + 2), -2),
    ({}, dict(factors=FAKE + 1), -2), ({"count": -1}, {}, -1), ({"count": 1 << 40}, {}, -1), ({"from": None}, {}, -1), ({"ld_from": 7}, {}, -1),
    ({"ld_to": 7}, {}, -1), ({"from_type": 3}, {}, -1), ({"to_type": 4}, {}, -1), ({"to_type": ops.F16}, {}, -1),
    ({"from_type": ops.F16, "to_type": ops.BF16}, {}, -1), ({"from_type": ops.F16}, {}, -1), ({"from": FAKE + 2}, {}, -2), ({"to": FAKE + 2}, {}, -2),
])
def test_clip_refuses(tensor, kw, code):
    assert B.lib().compams_clip_gradients(ctypes.byref(clip([tensor], **kw)), None) == code


@pytest.mark.parametrize("tensors,code", [
    ([{}, {}], -1),                                                         # the same tensor twice, in place
    ([{}, {"from": FAKE + 16, "to": FAKE + 16}], -1),                       # rows that overlap
    ([{"to": MORE}, {"from": LAST, "to": MORE}], -1), ([{"to": MORE}, {"from": MORE, "to": LAST}], -1), ([{"to": FAKE + 4}], -1),
    ([{"ld_to": 16}], -1),                                                  # in place with another stride
    ([{"to": None}, {"to": None}], -3), ([{"to": None}, {"to": MORE}], -3),  # read twice (what is refused is the workspace)
    ([{"ld_from": 16, "ld_to": 16}, {"from": FAKE + 32, "to": FAKE + 32, "ld_from": 16, "ld_to": 16}], -3),    # beside one another in rows
    ([{}, {"count": 0}], -3),
])
def test_clip_refuses_rows_that_are_written_twice(tensors, code):
    assert B.lib().compams_clip_gradients(ctypes.byref(clip(tensors, workspace_bytes=255)), None) == code


def test_null_and_workspace_sizes():
    L = B.lib()
    for call in (L.compams_gated_forward, L.compams_gated_backward, L.compams_projections_backward, L.compams_linear_cross_entropy,
                 L.compams_clip_gradients):
        assert call(None, None) == -1
    for size in (L.compams_gated_forward_workspace_size, L.compams_gated_backward_workspace_size, L.compams_projections_workspace_size,
                 L.compams_linear_loss_workspace_size, L.compams_clip_workspace_size):
        assert size(None) == 0
    # nothing is copied where rows start on 16 bytes
    assert L.compams_gated_forward_workspace_size(gated()) == 0
    assert L.compams_gated_forward_workspace_size(gated(n=1, rows=3, x=FAKE + 4)) == 0     # (nor is it for few rows)
    assert L.compams_gated_forward_workspace_size(gated(x=FAKE + 4)) > 0 and L.compams_gated_forward_workspace_size(gated(ld_gate_weight=17)) > 0
    assert L.compams_projections_workspace_size(projections()) == 0
    assert L.compams_projections_workspace_size(projections(ld_x=17)) > 0
    # the pieces of a vocabulary, whatever its size, are bounded
    large = dict(n=8, rows=1024, cols=768, type=ops.BF16, ld_x=768, ld_weight=768, ld_dx=768, ld_dweight=768, stride_dweight=1 << 30)
    for vocab in (50257, 500000):
        need = L.compams_linear_loss_workspace_size(linear_loss(vocab=vocab, **large))
        assert need < 8192 * 2 * vocab // 2
    assert L.compams_clip_workspace_size(ctypes.byref(clip([]))) == 256


def test_binding_refuses():
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    t = torch.zeros(4, dtype=torch.int64)
    for call in (lambda: ops.compams_gated_forward(x, w, w), lambda: ops.compams_gated_backward(x, x, x),
                 lambda: ops.compams_projections_backward(torch.zeros(4, 6), None, x, w, None), lambda: ops.compams_linear_cross_entropy(x, w, t),
                 lambda: ops.compams_clip_gradients(x, 1.0, 4)):     # host tensors
        with pytest.raises(ValueError):
            call()
    m = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="meta")  # noqa: E731
    for call in (lambda: ops.compams_gated_forward(m(4, 8), m(6, 8), m(6, 8), "tanh"), lambda: ops.compams_gated_forward(m(4, 8), m(6, 7), m(6, 8)),
                 lambda: ops.compams_gated_forward(m(4, 8), m(6, 8), m(5, 8)), lambda: ops.compams_gated_forward(m(4, 8), m(6, 8), m(6, 8, dtype=torch.float16)),
                 lambda: ops.compams_gated_forward(m(4, 8), m(6, 8), m(6, 8), gate=m(4, 6), keep=False),
                 lambda: ops.compams_gated_backward(m(4, 8), m(4, 8), m(4, 7)), lambda: ops.compams_gated_backward(m(5, 8), m(5, 8), m(5, 8), 2),
                 lambda: ops.compams_gated_backward(m(4, 8), m(4, 8), m(4, 8), accumulate=True),
                 lambda: ops.compams_gated_backward(m(4, 8), m(4, 8), m(4, 8), bias=False, dup_bias=m(1, 8)),
                 lambda: ops.compams_projections_backward(m(4, 6), None, None, None, None),
                 lambda: ops.compams_projections_backward(m(4, 6), None, m(4, 8), m(6, 8), m(6, 8)),
                 lambda: ops.compams_projections_backward(m(4, 6), m(4, 6), m(4, 8), None, m(6, 8)),
                 lambda: ops.compams_projections_backward(m(4, 6), m(4, 6), m(4, 8), m(6, 8), m(6, 8), accumulate=True),
                 lambda: ops.compams_projections_backward(m(4, 6), None, None, m(6, 8), None, dgate_weight=m(1, 6, 8)),
                 lambda: ops.compams_linear_cross_entropy(m(4, 8), m(6, 8), m(4)),
                 lambda: ops.compams_linear_cross_entropy(m(4, 8), m(6, 7), m(4, dtype=torch.int64)),
                 lambda: ops.compams_linear_cross_entropy(m(4, 8), m(6, 8), m(4, dtype=torch.int64), gradient=False, dx=m(4, 8)),
                 lambda: ops.compams_linear_cross_entropy(m(4, 8), m(6, 8), m(4, dtype=torch.int64), accumulate=True),
                 lambda: ops.compams_clip_gradients([], 1.0, 4), lambda: ops.compams_clip_gradients(m(4, 8), 1.0, 3),
                 lambda: ops.compams_clip_gradients([m(4, 8)], 1.0, 4, out=[m(4, 8), m(4, 8)]),
                 lambda: ops.compams_clip_gradients([m(4, 8)], 1.0, 4, out=[m(4, 7)])):
        with pytest.raises(ValueError):
            call()


def test_reference_bounds_hold_for_32_bits():
    """The bounds that the GPU tests use are wide enough for the same formulas in torch's fp32."""
    import product_reference as P
    g = torch.Generator().manual_seed(1)
    make = lambda r, c, s=1.0: torch.randn((r, c), generator=g) * s  # noqa: E731
    x, wg, wu, bg, bu = make(9, 33), make(7, 33, 0.2), make(7, 33, 0.2), make(1, 7)[0], make(1, 7)[0]
    for act in ops.ACTIVATIONS:
        a, b = x @ wg.t() + bg, x @ wu.t() + bu
        want, bound = P.gated_forward(x.double(), wg.double(), wu.double(), bg.double(), bu.double(), act, torch.float32)
        v, s, _, _ = P.activation(a, act)
        for got, w, o in zip((v * b, a, b), want, bound):
            P.close(got, w, o, act)
        dm = make(9, 7)
        want, bound = P.gated_backward(dm.double(), a.double(), b.double(), 3, act, torch.float32)
        for got, w, o in zip((dm * b * s, dm * v), want, bound):
            P.close(got, w, o, act)
    t = torch.tensor([1, 2, -100, 0, 6, 5, 3, 3, 2])
    want, bound = P.linear_cross_entropy(x.double(), wg.double(), t, 3, -100, 1.0, torch.float32)
    leaf, w = x.clone().requires_grad_(True), wg.clone().requires_grad_(True)
    loss = torch.nn.functional.cross_entropy(leaf @ w.t(), t, reduction="none")
    count = (t != -100).reshape(3, 3).sum(1)
    (loss.reshape(3, 3).sum(1) / count).sum().backward()
    P.close(loss, want[1], bound[1], "losses")
    P.close(leaf.grad, want[2], bound[2], "dx")
    P.close(w.grad, want[3].sum(0), bound[3].sum(0), "dweight")


def test_registers_of_the_kernels():
    """No more than eight registers of a lane are spilled, and where three workgroups are to share a compute unit, three fit."""
    pytest.importorskip("msgpack")
    import re
    import test_operator_kernels_cpu as K
    found = {}
    for elf in K.code_objects(open(B.LIB_PATH, "rb").read()):
        found.update(K.kernels(elf))
    ours = {k: v for k, v in found.items() if re.search(r"k_(gated|projection|linear_loss|clip|pack)", k)}
    assert len(ours) > 100
    over = {k: v[".vgpr_spill_count"] for k, v in ours.items() if v[".vgpr_spill_count"] > 8}
    assert not over, over
    three = {k: v[".vgpr_count"] for k, v in ours.items() if "linear_loss_piece" in k and "DF16" in k and v[".group_segment_fixed_size"] == 49152}
    assert len(three) == 2 and max(three.values()) <= 168, three
