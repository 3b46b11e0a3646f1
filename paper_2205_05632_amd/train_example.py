"""A whole training step on one GPU: a small residual next-token model, n workers with their own tokens, dropout, layer norms,
the loss, and Algorithm 2 on their gradients.

    python -m paper_2205_05632_amd.train_example [--workers 4] [--steps 60] [--dropout 0.1] [--compressor topk]

The model is a tied embedding of V tokens, `layers` blocks

    y = LN(h),   h' = h + dropout(relu(y W1 + b1) W2 + b2)

and a last norm in front of the embedding as output layer.  Its parameters are views of the optimizer's flat theta and
their gradients views of the workers' rows of g, where compams_step reads them.  torch does the matrix products (in
bfloat16, the residual stream stays in float32); everything between them is the library's: the join of a block's end
with the next block's norm, the cross-entropy, their gradients, and the step.  Tokens follow a random first-order chain,
so that there is something to learn.  Prints one JSON line.
"""
import argparse
import json
import math

import torch

from . import binding as B
from . import operators as ops


class Model:
    """Shapes and places of the parameters in the flat vector."""

    def __init__(self, vocab: int = 512, width: int = 256, hidden: int = 768, layers: int = 2):
        self.vocab, self.width, self.hidden, self.layers = vocab, width, hidden, layers
        shapes = [("embed", (vocab, width))]
        for i in range(layers):
            shapes += [(f"gamma{i}", (width,)), (f"beta{i}", (width,)), (f"w1_{i}", (width, hidden)), (f"b1_{i}", (hidden,)),
                       (f"w2_{i}", (hidden, width)), (f"b2_{i}", (width,))]
        shapes += [(f"gamma{layers}", (width,)), (f"beta{layers}", (width,))]
        self.place, first = {}, 0
        for name, shape in shapes:
            self.place[name] = (first, shape)
            first += math.prod(shape)
        self.d = first

    def views(self, flat: torch.Tensor):
        """The parameters in a vector of d entries."""
        return {k: flat[a:a + math.prod(s)].view(s) for k, (a, s) in self.place.items()}

    def vectors(self, rows: torch.Tensor, name: str):
        """A one-dimensional parameter's gradients in the workers' rows: n x its size."""
        a, (size,) = self.place[name]
        return rows[:, a:a + size]

    def initial(self, seed: int = 0) -> torch.Tensor:
        g = torch.Generator().manual_seed(seed)
        flat = torch.zeros(self.d)
        for name, p in self.views(flat).items():
            if name.startswith("gamma"):
                p.fill_(1.0)
            elif p.dim() == 2:
                fan, scale = (p.shape[1], 0.5) if name == "embed" else (p.shape[0], 1.0)
                p.copy_(torch.randn(p.shape, generator=g) * scale / math.sqrt(fan))
        return flat


def forward_backward(model: Model, theta: torch.Tensor, tokens: torch.Tensor, targets: torch.Tensor, g: torch.Tensor, p: float,
                     seed: int, step: int, dtype=torch.bfloat16) -> torch.Tensor:
    """Fills the workers' rows of g (n x ld) with the gradients of their mean losses and returns those (n).  tokens and
    targets: n x tokens of a worker."""
    n, rows = tokens.shape
    w = model.views(theta)
    low = {k: v.to(dtype) for k, v in w.items() if v.dim() == 2}
    flat, layers = tokens.reshape(-1), model.layers
    join = lambda x, h, i, bias: ops.compams_dropout_add_norm_forward(  # noqa: E731
        x, h, w[f"gamma{i}"], w[f"beta{i}"], p, seed, step * (layers + 1) + i, bias=bias,
        h=torch.empty(x.shape, dtype=torch.float32, device=x.device))
    h, y, mean, rstd = join(low["embed"][flat], None, 0, None)
    kept = [(h, y, mean, rstd)]
    middles = []
    for i in range(layers):
        m = torch.relu_(torch.addmm(w[f"b1_{i}"].to(dtype), y, low[f"w1_{i}"]))
        h, y, mean, rstd = join(m @ low[f"w2_{i}"], h, i + 1, w[f"b2_{i}"])
        kept.append((h, y, mean, rstd))
        middles.append(m)
    logits = y @ low["embed"].t()
    loss, _, dlogits = ops.compams_cross_entropy(logits, targets.reshape(-1), n, dlogits=logits)

    grads = [model.views(g[k]) for k in range(n)]
    of = lambda t, k: t[k * rows:(k + 1) * rows]  # noqa: E731
    for k in range(n):
        grads[k]["embed"].copy_(of(dlogits, k).t() @ of(y, k))
    dy, dh = dlogits @ low["embed"], None
    for i in range(layers, -1, -1):
        h, _, mean, rstd = kept[i]
        bias = {} if i == 0 else {"dbias": model.vectors(g, f"b2_{i - 1}")}
        dx, dh, _, _, _ = ops.compams_dropout_add_norm_backward(
            dy, dh, h, mean, rstd, w[f"gamma{i}"], p, seed, step * (layers + 1) + i, n,
            dgamma=model.vectors(g, f"gamma{i}"), dbeta=model.vectors(g, f"beta{i}"), **bias)
        if i == 0:
            break
        m = middles[i - 1]
        da = (dx @ low[f"w2_{i - 1}"].t()).masked_fill_(m == 0, 0.0)
        for k in range(n):
            grads[k][f"w2_{i - 1}"].copy_(of(m, k).t() @ of(dx, k))
            grads[k][f"w1_{i - 1}"].copy_(of(kept[i - 1][1], k).t() @ of(da, k))
            torch.sum(of(da, k), 0, dtype=torch.float32, out=grads[k][f"b1_{i - 1}"])
        dy = da @ low[f"w1_{i - 1}"].t()
    for k in range(n):
        grads[k]["embed"].index_add_(0, tokens[k], of(dx, k).float())
    return loss


def chain(model: Model, n: int, rows: int, step: int, device, seed: int = 7):
    """Tokens of a first-order chain in which every token has four likely successors."""
    g = torch.Generator(device=device).manual_seed(seed)
    after = torch.randint(0, model.vocab, (model.vocab, 4), generator=g, device=device)
    g.manual_seed(seed * 1000003 + step + 1)
    t = torch.randint(0, model.vocab, (n, rows), generator=g, device=device)
    choice = torch.randint(0, 4, (n, rows), generator=g, device=device)
    return t, after[t, choice]


def train(workers: int = 4, rows: int = 512, steps: int = 60, p: float = 0.1, compressor: str = "topk", lr: float = 2e-3,
          model: Model = None, device="cuda:0"):
    """Losses (steps x workers)."""
    model = model or Model()
    if compressor == "topk":
        kw = dict(compressor=B.TOPK, k=max(1, model.d // 20))
    elif compressor == "none":
        kw = dict(compressor=B.NONE)
    else:
        raise ValueError(f"unknown compressor {compressor!r}")
    opt = B.Compams(workers, model.d, model.initial(), device=device, **kw)
    g = torch.zeros((workers, opt.ld), device=opt.device)
    losses = []
    for step in range(steps):
        tokens, targets = chain(model, workers, rows, step, opt.device)
        losses.append(forward_backward(model, opt.theta, tokens, targets, g, p, seed=1, step=step))
        opt.compams_step(g, lr)
    out = torch.stack(losses)
    opt.close()
    return out


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--compressor", choices=["topk", "none"], default="topk")
    args = ap.parse_args()
    losses = train(args.workers, steps=args.steps, p=args.dropout, compressor=args.compressor).mean(1).tolist()
    print(json.dumps({"steps": args.steps, "workers": args.workers, "first_loss": losses[0], "last_loss": losses[-1]}))


if __name__ == "__main__":
    main()
