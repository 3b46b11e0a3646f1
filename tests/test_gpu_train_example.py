"""The small training program that runs the operators and the optimizer step together."""
import pytest
import torch

import operator_reference as R
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
        m = torch.relu(norm(h, i) @ w[f"w1_{i}"] + w[f"b1_{i}"])
        h = h + drop(m @ w[f"w2_{i}"] + w[f"b2_{i}"], i + 1)
    logits = norm(h, model.layers) @ w["embed"].t()
    return torch.nn.functional.cross_entropy(logits, targets.reshape(-1), reduction="none").reshape(n, rows).mean(1)


def test_gradients_of_the_whole_model():
    """Every worker's row against autograd in 64 bits on the host, with the same dropout masks."""
    model = T.Model(vocab=61, width=40, hidden=56, layers=2)
    n, rows, p, seed, step = 3, 17, 0.2, 11, 4
    g = torch.Generator().manual_seed(2)
    theta = model.initial(3)
    theta += 0.05 * torch.randn(model.d, generator=g)
    tokens = torch.randint(0, 61, (n, rows), generator=g)
    targets = torch.randint(0, 61, (n, rows), generator=g)
    grad = torch.full((n, model.d + 12), 5.0, device="cuda")
    loss = T.forward_backward(model, theta.cuda(), tokens.cuda(), targets.cuda(), grad, p, seed, step, torch.float32)
    leaf = theta.double().requires_grad_(True)
    want = reference_loss(model, leaf, tokens, targets, p, seed, step)
    assert torch.allclose(loss.cpu().double(), want.detach(), rtol=1e-5)
    for k in range(n):
        (row,) = torch.autograd.grad(want[k], leaf, retain_graph=True)
        # fp32 products over at most 56 + 61 terms and a chain of seven of them: far below 1e-4 of the largest entry
        assert float((grad[k, :model.d].cpu().double() - row).abs().max()) <= 1e-4 * float(row.abs().max())
    assert bool((grad[:, model.d:] == 5.0).all())


@pytest.mark.parametrize("compressor", ["topk", "none"])
def test_the_loss_falls(compressor):
    """Sixty steps of four workers: from log 512 = 6.2 to well below it (the chain's own entropy is log 4 = 1.4)."""
    losses = T.train(steps=60, compressor=compressor).mean(1).cpu()
    assert bool(torch.isfinite(losses).all())
    assert 5.5 < float(losses[0]) < 8.0 and float(losses[-5:].mean()) < float(losses[0]) - 1.0
