"""Host-only checks of the operators' boundary: the binding's structures, the generator's published vectors, and what the
entry points refuse before anything is enqueued (no GPU needed)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import operator_reference as R
from paper_2205_05632_amd import binding as B
from paper_2205_05632_amd import operators as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name", ["compams_drop", "compams_norm", "compams_loss"])
def test_structures_match_the_header(tmp_path, name):
    struct = getattr(ops, name)
    fields = [f[0] for f in struct._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "compams.h"\nint main(void){\n'
                   + f'printf("%zu\\n", sizeof({name}));\n'
                   + "".join(f'printf("%zu\\n", offsetof({name}, {f}));\n' for f in fields) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert out[0] == ctypes.sizeof(struct)
    assert out[1:] == [getattr(struct, f).offset for f in fields]


@pytest.mark.parametrize("name", ["drop", "norm", "loss"])
def test_packed_arguments_have_the_structures_layout(name):
    packer, struct = getattr(ops, "_" + name.upper()), getattr(ops, "compams_" + name)
    leaves = []

    def walk(s, base):
        for field, kind in s._fields_:
            at = base + getattr(s, field).offset
            if issubclass(kind, ctypes.Structure):
                walk(kind, at)
            else:
                leaves.append((at, kind))

    walk(struct, 0)
    assert packer.size == ctypes.sizeof(struct)
    values = [i + 1.5 if kind in (ctypes.c_float, ctypes.c_double) else i + 1 for i, (_, kind) in enumerate(leaves)]
    raw = packer.pack(*values)
    assert [kind.from_buffer_copy(raw, at).value for at, kind in leaves] == values


def test_generator_of_the_reference():
    """The vectors published with the generator (Salmon, Moraes, Dror, Shaw 2011), and both forms against each other."""
    assert R.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert R.philox((ones,) * 4, (ones, ones)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    seed, offset = 0x0123456789ABCDEF, 0xFEDCBA9876543210
    u = R.numbers(3, 21, seed, offset)
    for r, c in ((0, 0), (1, 7), (2, 8), (2, 20)):
        w = R.philox((c // 8, r, offset & ones, offset >> 32), (seed & ones, seed >> 32))
        assert u[r, c] == (w[c % 8 // 2] >> (16 * (c % 2))) & 0xFFFF


FAKE = 0x1000    # never dereferenced: validation fails first


def norm(**kw):
    a = ops.compams_norm(n=2, rows=3, cols=8, type=ops.F32, stream_type=ops.F32, eps=1e-5, h=FAKE, ld_h=8, y=FAKE, ld_y=8,
                         x=None, ld_x=8, mean=FAKE, rstd=FAKE, dy=FAKE, ld_dy=8)
    for k, v in kw.items():
        if k in ("p", "seed", "offset", "step"):
            setattr(a.drop, k, v)
        else:
            setattr(a, k, v)
    return ctypes.byref(a)


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), -1), (dict(n=65536), -1), (dict(rows=-1), -1), (dict(rows=1 << 31), -1), (dict(n=65535, rows=65535), -1),
    (dict(cols=0), -1), (dict(cols=1 << 31), -1), (dict(type=3), -1), (dict(type=-1), -1), (dict(type=ops.F32, stream_type=ops.F16), -1),
    (dict(type=ops.F16, stream_type=ops.BF16), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
    (dict(eps=float("inf")), -1), (dict(h=None), -1), (dict(y=None), -1), (dict(ld_h=7), -1), (dict(ld_y=0), -1),
    (dict(h=FAKE + 2), -2), (dict(y=FAKE + 1), -2), (dict(gamma=FAKE + 2), -2), (dict(mean=FAKE + 3), -2), (dict(x=FAKE), -1),
])
def test_layer_norm_forward_refuses(kw, code):
    assert B.lib().compams_layer_norm_forward(norm(**kw), None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), -1), (dict(p=1.5), -1), (dict(p=-0.5), -1), (dict(p=float("nan")), -1), (dict(step=FAKE + 4), -2),
    (dict(ld_x=7), -1), (dict(x=FAKE + 2), -2), (dict(residual=FAKE, ld_residual=7), -1), (dict(bias=FAKE + 1), -2),
])
def test_join_forward_refuses(kw, code):
    assert B.lib().compams_dropout_add_norm_forward(norm(**dict(dict(x=FAKE), **kw)), None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dresidual=None), -1), (dict(dy=None), -1), (dict(mean=None), -1), (dict(rstd=None), -1), (dict(h=None), -1),
    (dict(ld_dy=7), -1), (dict(ld_dresidual=7), -1), (dict(dresidual=FAKE + 2), -2), (dict(accumulate=2), -1),
    (dict(dgamma=FAKE, ld_dgamma=7), -1), (dict(dgamma=FAKE + 2, ld_dgamma=8), -2), (dict(n=0), -1), (dict(rows=-5), -1),
    (dict(rows=100000, dgamma=FAKE, ld_dgamma=8), -1), (dict(rows=100000, dgamma=FAKE, ld_dgamma=8, workspace=FAKE, workspace_bytes=256), -3),
    (dict(rows=100000, dgamma=FAKE, ld_dgamma=8, workspace=FAKE + 16, workspace_bytes=1 << 30), -2),
    (dict(cols=100000, ld_h=100000, ld_dy=100000, ld_dresidual=100000), -1),
])
def test_backward_refuses(kw, code):
    kw = dict(dict(dresidual=FAKE, ld_dresidual=8), **kw)
    assert B.lib().compams_layer_norm_backward(norm(**kw), None) == code
    assert B.lib().compams_dropout_add_norm_backward(norm(**kw), None) == code


def test_layer_norm_backward_takes_no_branch():
    for extra in ("dx", "dh", "dbias"):
        kw = {extra: FAKE, "ld_" + extra: 8}
        assert B.lib().compams_layer_norm_backward(norm(dresidual=FAKE, ld_dresidual=8, **kw), None) == -1


def test_null_and_workspace_sizes():
    L = B.lib()
    for call in (L.compams_layer_norm_forward, L.compams_layer_norm_backward, L.compams_dropout_add_norm_forward,
                 L.compams_dropout_add_norm_backward, L.compams_cross_entropy):
        assert call(None, None) == -1
    assert L.compams_norm_workspace_size(None) == 0 and L.compams_loss_workspace_size(None) == 0
    assert L.compams_norm_workspace_size(norm(n=0, dgamma=FAKE)) == 0
    many = L.compams_norm_workspace_size(norm(n=8, rows=8192, cols=768, dgamma=FAKE))
    assert 0 < many < 64 << 20 and many % 256 == 0
    # an empty call needs nothing and does nothing
    assert L.compams_layer_norm_forward(norm(rows=0), None) == 0


def drop(**kw):
    d = ops.compams_drop(0.5, 1, 2, None)
    for k, v in kw.items():
        setattr(d, k, v)
    return ctypes.byref(d)


@pytest.mark.parametrize("args,code", [
    ((0, 3, 8, 0, 0, FAKE, 8, None, 0, FAKE, 8, drop(), None), -1),
    ((1, -3, 8, 0, 0, FAKE, 8, None, 0, FAKE, 8, drop(), None), -1),
    ((1, 3, 0, 0, 0, FAKE, 8, None, 0, FAKE, 8, drop(), None), -1),
    ((1, 3, 8, 4, 0, FAKE, 8, None, 0, FAKE, 8, drop(), None), -1),
    ((1, 3, 8, 1, 2, FAKE, 8, None, 0, FAKE, 8, drop(), None), -1),
    ((1, 3, 8, 0, 0, None, 8, None, 0, FAKE, 8, drop(), None), -1),
    ((1, 3, 8, 0, 0, FAKE, 8, None, 0, None, 8, drop(), None), -1),
    ((1, 3, 8, 0, 0, FAKE, 7, None, 0, FAKE, 8, drop(), None), -1),
    ((1, 3, 8, 0, 0, FAKE, 8, FAKE, 7, FAKE, 8, drop(), None), -1),
    ((1, 3, 8, 0, 0, FAKE, 8, None, 0, FAKE, 8, None, None), -1),
    ((1, 3, 8, 0, 0, FAKE, 8, None, 0, FAKE, 8, drop(p=1.01), None), -1),
    ((1, 3, 8, 0, 0, FAKE + 2, 8, None, 0, FAKE, 8, drop(), None), -2),
    ((1, 3, 8, 0, 0, FAKE, 8, None, 0, FAKE, 8, drop(step=FAKE + 4), None), -2),
    ((1, 0, 8, 0, 0, None, 8, None, 0, None, 8, drop(), None), 0),
])
def test_dropout_refuses(args, code):
    assert B.lib().compams_dropout(*args) == code


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), -1), (dict(rows=-1), -1), (dict(vocab=0), -1), (dict(vocab=1 << 31), -1), (dict(type=ops.I32), -1),
    (dict(target_type=ops.F32), -1), (dict(logits=None), -1), (dict(targets=None), -1), (dict(ld_logits=7), -1),
    (dict(ld_dlogits=7), -1), (dict(workspace=None), -1), (dict(workspace=FAKE + 16), -2), (dict(workspace_bytes=8), -3),
    (dict(targets=FAKE + 4), -2), (dict(logits=FAKE + 2), -2), (dict(dlogits=FAKE + 2), -2), (dict(losses=FAKE + 2), -2),
    (dict(mean_loss=None, losses=None, dlogits=None), -1),
])
def test_cross_entropy_refuses(kw, code):
    a = ops.compams_loss(n=2, rows=3, vocab=8, type=ops.F32, target_type=ops.I64, logits=FAKE, ld_logits=8, targets=FAKE,
                         grad_scale=1.0, mean_loss=FAKE, losses=FAKE, dlogits=FAKE, ld_dlogits=8, workspace=FAKE,
                         workspace_bytes=1 << 20)
    for k, v in kw.items():
        setattr(a, k, v)
    assert B.lib().compams_cross_entropy(ctypes.byref(a), None) == code


def test_binding_refuses_host_tensors_and_other_types():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        ops.compams_layer_norm_forward(x, None, None)
    with pytest.raises(ValueError):
        ops.compams_dropout(x, 0.5, 1)
    with pytest.raises(ValueError):
        ops.compams_cross_entropy(x, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        ops.compams_dropout(x.to(torch.int32), 0.5, 1)


def test_reference_bounds_hold_for_32_bits():
    """The bounds that the GPU tests use are wide enough for the same formulas in torch's fp32."""
    rng = np.random.default_rng(1)
    h = torch.from_numpy(rng.standard_normal((5, 301))).float()
    one, zero = torch.ones(301), torch.zeros(301)
    want, bound = R.norm_forward(h.double(), one.double(), zero.double(), 1e-5, torch.float32)
    mean = h.mean(1)
    rstd = 1 / torch.sqrt((h - mean[:, None]).square().mean(1) + 1e-5)
    for got, w, b in zip(((h - mean[:, None]) * rstd[:, None], mean, rstd), want, bound):
        R.close(got, w, b, "forward")
    x = torch.from_numpy(rng.standard_normal((6, 77)) * 3).float()
    t = torch.from_numpy(rng.integers(0, 77, 6))
    want, bound = R.cross_entropy(x.double(), t, 2, -100, 1.0, torch.float32)
    leaf = x.clone().requires_grad_(True)
    loss = torch.nn.functional.cross_entropy(leaf, t, reduction="none")
    (loss.sum() / 3).backward()
    R.close(loss, want[1], bound[1], "losses")
    R.close(leaf.grad, want[2], bound[2], "dlogits")
