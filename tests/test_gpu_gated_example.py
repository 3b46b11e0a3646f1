"""The training program with gated blocks, an output layer whose logits are never stored, and clipped gradients."""
import json
import math
import subprocess
import sys

import pytest
import torch

import operator_reference as R
from paper_2205_05632_amd import operators as ops
from paper_2205_05632_amd import train_example as T

pytestmark = pytest.mark.gpu


def reference_loss(model, theta, tokens, targets, p, seed, step):
    """A worker's mean loss, in the dtype of theta, by torch's own operations (differentiable)."""
    n, rows = tokens.shape
    w = model.views(theta)
    keeps = lambda i: R.kept(n * rows, model.width, p, seed, step * (model.layers + 1) + i)  # noqa: E731
    drop = lambda x, i: torch.where(keeps(i), x * R.factor(p), 0.0)  # noqa: E731
    norm = lambda h, i: torch.nn.functional.layer_norm(h, (model.width,), w[f"gamma{i}"], w[f"beta{i}"], 1e-5)  # noqa: E731
    h = drop(w["embed"][tokens.reshape(-1)], 0)
    for i in range(model.layers):
        y = norm(h, i)
        m = torch.nn.functional.silu(y @ w[f"wg_{i}"].t() + w[f"bg_{i}"]) * (y @ w[f"wu_{i}"].t() + w[f"bu_{i}"])
        h = h + drop(m @ w[f"wd_{i}"].t() + w[f"b2_{i}"], i + 1)
    logits = norm(h, model.layers) @ w["embed"].t()
    return torch.nn.functional.cross_entropy(logits, targets.reshape(-1), reduction="none").reshape(n, rows).mean(1)


def test_gradients_of_the_whole_model():
    """Every worker's row against autograd in 64 bits on the host, with the same dropout masks; then cut to a norm."""
    model = T.Model(vocab=61, width=40, hidden=56, layers=2, gated=True)
    n, rows, p, seed, step = 3, 17, 0.2, 11, 4
    g = torch.Generator().manual_seed(2)
    theta = model.initial(3)
    theta += 0.05 * torch.randn(model.d, generator=g)
    tokens = torch.randint(0, 61, (n, rows), generator=g)
    targets = torch.randint(0, 61, (n, rows), generator=g)
    grad = torch.full((n, model.d + 12), 5.0, device="cuda")
    loss = T.forward_backward_gated(model, theta.cuda(), tokens.cuda(), targets.cuda(), grad, p, seed, step, torch.float32)
    leaf = theta.double().requires_grad_(True)
    want = reference_loss(model, leaf, tokens, targets, p, seed, step)
    assert torch.allclose(loss.cpu().double(), want.detach(), rtol=1e-5)
    exact = [torch.autograd.grad(want[k], leaf, retain_graph=True)[0] for k in range(n)]
    for k, row in enumerate(exact):
        # fp32 products over at most 61 terms and a chain of nine of them: far below 1e-4 of the largest entry
        assert float((grad[k, :model.d].cpu().double() - row).abs().max()) <= 1e-4 * float(row.abs().max())
    assert bool((grad[:, model.d:] == 5.0).all())
    size = torch.stack([row.norm() for row in exact])
    largest = float(size.median())
    before = grad.clone()
    _, norms, factors = ops.compams_clip_gradients(grad[:, :model.d], largest, n)
    assert torch.allclose(norms.cpu().double(), size, rtol=1e-4)
    assert torch.allclose(factors.cpu().double(), (largest / size).clamp(max=1.0), rtol=1e-4)
    assert torch.equal(grad[:, :model.d], before[:, :model.d] * factors[:, None]) and bool((grad[:, model.d:] == 5.0).all())


@pytest.mark.parametrize("compressor", ["topk", "none"])
def test_training_runs(compressor):
    losses = T.train(steps=6, compressor=compressor, model=T.Model(gated=True), clip=1.0)
    assert losses.shape == (6, 4) and bool(torch.isfinite(losses).all())


def test_the_command():
    out = subprocess.run([sys.executable, "-m", "paper_2205_05632_amd.train_example", "--gated", "--clip", "1.0", "--steps", "3"],
                         capture_output=True, text=True, timeout=100, check=True)
    said = json.loads(out.stdout.strip().splitlines()[-1])
    assert said["steps"] == 3 and math.isfinite(said["last_loss"])
