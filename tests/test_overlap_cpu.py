"""Host-only checks of what calls of the operators with products refuse: outputs that lie over inputs, or over one another, where a
kernel would read what another workgroup has written.  (The pointers are never dereferenced: these calls end before anything is enqueued.)"""
import ctypes
import os
import subprocess

import pytest

from paper_2205_05632_amd import binding as B
from paper_2205_05632_amd import operators as ops

HERE = os.path.dirname(os.path.abspath(__file__))
MB = 1 << 20
ROOM = dict(workspace=1 << 40, workspace_bytes=1 << 38)


def at(place, shift=0):
    """A buffer of its own for every place, 16 MB apart."""
    return (16 * place + 16) * MB + shift


def test_areas_against_their_bytes(tmp_path):
    """Every pair of small areas: none that share a byte is missed, and of equal distances none is taken to that does not."""
    out = str(tmp_path / "model")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(os.path.dirname(HERE), "paper_2205_05632_amd", "csrc"),
                    os.path.join(HERE, "areas_model.cpp"), "-o", out], check=True)
    r = subprocess.run([out], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


def backward(**kw):
    a = ops.compams_gated(n=2, rows=300, hidden=8, type=ops.F32, activation=0, dm=at(0), ld_dm=8, gate=at(1), ld_gate=8, up=at(2), ld_up=8,
                          dgate=at(3), ld_dgate=8, dup=at(4), ld_dup=8, dgate_bias=at(5), ld_dgate_bias=8, dup_bias=at(6), ld_dup_bias=8, **ROOM)
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


@pytest.mark.parametrize("kw", [
    dict(dgate=at(1), ld_dgate=16),                                     # over gate with another distance from row to row
    dict(dup=at(0), ld_dup=16), dict(dgate=at(2), ld_dgate=9),
    dict(dgate=at(1, 32)), dict(dup=at(2, -32)), dict(dgate=at(0, 16)),  # a row further, a row before, a part of one
    dict(dgate=at(4, 32)), dict(dup=at(3, 299 * 32)),                   # over one another
    dict(dgate_bias=at(6, 32)), dict(dgate_bias=at(0, 64)), dict(dup_bias=at(4, 160)),
    dict(gate=at(1), ld_gate=24, dgate=at(1, 28), ld_dgate=24),          # beside gate's columns, but for one
])
def test_gated_backward_refuses_outputs_over_inputs(kw):
    assert B.lib().compams_gated_backward(backward(**kw), None) == -1


def forward(**kw):
    a = ops.compams_gated(n=2, rows=300, cols=16, hidden=8, type=ops.F32, activation=0, x=at(0), ld_x=16, gate_weight=at(1), ld_gate_weight=16,
                          up_weight=at(2), ld_up_weight=16, gate_bias=at(3), up_bias=at(4), m=at(5), ld_m=8, gate=at(6), ld_gate=8, up=at(7),
                          ld_up=8, **ROOM)
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


@pytest.mark.parametrize("kw", [
    dict(m=at(0)), dict(m=at(0), ld_m=16), dict(gate=at(0), ld_gate=16), dict(up=at(0, 32), ld_up=16),     # x
    dict(n=1, rows=1, m=at(0)), dict(n=1, rows=1, gate=at(1)),           # a token
    dict(m=at(1)), dict(up=at(2, 7 * 64)), dict(gate=at(3, 28)), dict(m=at(4)),
    dict(m=at(6, 32)), dict(gate=at(7, 599 * 32)), dict(up=at(5, 4)),    # one another
])
def test_gated_forward_refuses_outputs_over_inputs(kw):
    assert B.lib().compams_gated_forward(forward(**kw), None) == -1


def projections(**kw):
    a = ops.compams_projections(n=2, rows=300, cols=16, hidden=8, type=ops.F32, dgate=at(0), ld_dgate=8, dup=at(1), ld_dup=8, x=at(2), ld_x=16,
                                gate_weight=at(3), ld_gate_weight=16, up_weight=at(4), ld_up_weight=16, dx=at(5), ld_dx=16,
                                dgate_weight=at(6), ld_dgate_weight=16, stride_dgate_weight=1024, dup_weight=at(7), ld_dup_weight=16,
                                stride_dup_weight=1024, **ROOM)
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


@pytest.mark.parametrize("kw", [
    dict(dx=at(0)), dict(dx=at(0), ld_dx=32), dict(dx=at(1)), dict(dx=at(2)), dict(dx=at(2, 64)), dict(dx=at(3)), dict(dx=at(4, 64)),
    dict(dx=at(6)), dict(dx=at(7, 4096)), dict(dgate_weight=at(0)), dict(dup_weight=at(2)), dict(dgate_weight=at(4)),
    dict(dup_weight=at(6, 7 * 64)), dict(dup_weight=at(6, 4096)), dict(dgate_weight=at(7, 4096 + 60)),      # one another's, of one worker or two
    dict(ld_dgate_weight=32, ld_dup_weight=32, dup_weight=at(6, 60)),    # beside one another's columns, but for one
    dict(dup=None, up_weight=None, dup_weight=None, dx=at(0)), dict(dup=None, up_weight=None, dup_weight=None, dgate_weight=at(2)),
])
def test_projections_refuse_outputs_over_inputs(kw):
    assert B.lib().compams_projections_backward(projections(**kw), None) == -1


def linear_loss(**kw):
    a = ops.compams_linear_loss(n=2, rows=300, cols=16, vocab=50, type=ops.F32, target_type=ops.I64, x=at(0), ld_x=16, weight=at(1), ld_weight=16,
                                targets=at(2), grad_scale=1.0, mean_loss=at(3), losses=at(4), dx=at(5), ld_dx=16, dweight=at(6), ld_dweight=16,
                                stride_dweight=1024, **ROOM)
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


@pytest.mark.parametrize("kw", [
    dict(dx=at(1)), dict(dx=at(1, 49 * 64)), dict(dx=at(1), ld_dx=32), dict(dx=at(2)), dict(dx=at(6, 4096)), dict(dweight=at(0)),
    dict(dweight=at(1)), dict(dweight=at(1, -64)), dict(dweight=at(2, 8)), dict(losses=at(0, 4)), dict(losses=at(2)), dict(mean_loss=at(4, 4)),
    dict(mean_loss=at(1)), dict(losses=at(5)), dict(dx=at(4, -599 * 64)),
])
def test_linear_cross_entropy_refuses_outputs_over_inputs(kw):
    assert B.lib().compams_linear_cross_entropy(linear_loss(**kw), None) == -1


def clip(n, **kw):
    t = ops.compams_clip_tensor(**{"from": at(0), "ld_from": 100, "to": at(1), "ld_to": 100, "count": 40, "from_type": ops.F32,
                                   "to_type": ops.F32, **kw})
    a = ops.compams_clip(n=n, tensors=1, tensor=ctypes.addressof(t), max_norm=1.0, scale=1.0, norms=at(2), factors=at(3), workspace=at(4),
                         workspace_bytes=255)
    a.table = t
    return a


@pytest.mark.parametrize("n,kw,code", [
    (3, {"to": at(0, 400)}, -1), (3, {"to": at(0, -800)}, -1), (3, {"to": at(0, 2 * 400 + 156)}, -1), (3, {"to": at(0, 300)}, -1),
    (4, {"to": at(0, 800), "ld_to": 50}, -1), (2, {"from_type": ops.F16, "to": at(0, 200)}, -1),
    # side by side, behind one another, of one worker (what is refused is the workspace)
    (3, {"to": at(0, 160)}, -3), (3, {"to": at(0, 400 + 240)}, -3), (3, {"to": at(0, 1200)}, -3), (1, {"to": at(0, 400)}, -3),
    (3, {"to": at(0, 160), "ld_to": 200}, -3), (3, {}, -3),
])
def test_clip_refuses_rows_over_another_workers(n, kw, code):
    assert B.lib().compams_clip_gradients(ctypes.byref(clip(n, **kw)), None) == code
