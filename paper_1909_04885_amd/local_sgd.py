"""Local SGD on categorical rows with many classes (Section 2.2 and Section 5.1 "lSGD": every solver makes H steps of its own
on the samples of its chunks, starting from the shared model, and the trainer merges the models, weighted by samples).

The model: a row's token is looked up in a table, scaled by the square root of its width, normalised, and scored against
all classes.  A step of a solver runs every training operator of the library: lookup, layer norm, softmax loss with its
gradients, the gradients of layer norm and lookup, and clipping by their common norm.  Solvers own whole chunks, dealt
by `balance`, as in the CoCoA round; on one GPU they run one after the other, each from the same shared model.

    python -m paper_1909_04885_amd.local_sgd --rows 65536 --tokens 20000 --classes 5000 --width 256 --solvers 4 --rounds 8
"""
from __future__ import annotations

import argparse
import json
import math
import sys
import time
from typing import Dict, List, Sequence

from .binding import balance
from .train import TrainOps

TYPES = ("float32", "bfloat16", "float16")


class TokenModel:
    """table [tokens, width], gamma and beta [width], weights [classes, width]: one type, 32-bit masters for the merge."""

    def __init__(self, tokens: int, classes: int, width: int, dtype, device: str, seed: int = 0):
        import torch
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        spread = 1.0 / math.sqrt(width)
        self.master = [torch.randn(tokens, width, generator=gen, device=device) * spread, torch.ones(width, device=device),
                       torch.zeros(width, device=device), torch.randn(classes, width, generator=gen, device=device) * spread]
        self.dtype = dtype
        self.scale = math.sqrt(width)


def loss_and_gradients(ops: TrainOps, params: Sequence, scale: float, tokens, labels, row_weight):
    """(loss of every row, gradients in the order of the parameters) of sum_i row_weight_i loss_i."""
    table, gamma, beta, weights = params
    x = ops.embed(table, tokens, scale)
    y, mean, rstd = ops.layer_norm(x, gamma, beta)
    loss, dy, dweights = ops.softmax_loss_grad(y, weights, labels, row_weight)
    dx, dgamma, dbeta = ops.layer_norm_grad(dy, x, gamma, mean, rstd)
    return loss, [ops.embed_grad(tokens, dx, table.shape[0], scale), dgamma, dbeta, dweights]


def evaluate(ops: TrainOps, model: TokenModel, tokens, labels, batch: int = 8192) -> float:
    """Mean loss over the rows with a label."""
    table, gamma, beta, weights = [p.to(model.dtype) for p in model.master]
    total = 0.0
    for i in range(0, tokens.shape[0], batch):
        y, _, _ = ops.layer_norm(ops.embed(table, tokens[i:i + batch], model.scale), gamma, beta)
        total += float(ops.softmax_loss(y, weights, labels[i:i + batch])[0].double().sum())
    return total / max(1, int((labels >= 0).sum()))


def step_rows(step: int, batch: int, n: int, device=None):
    """The rows of a solver's step, counted over all rounds: `batch` of its n rows after those of the step before, and from the first again."""
    import torch
    return torch.arange(step * batch, (step + 1) * batch, device=device) % n


def local_steps(ops: TrainOps, model: TokenModel, tokens, labels, steps: int, batch: int, rate: float, momentum: float, max_norm: float,
                loss_scale: float, first: int = 0) -> List:
    """H = `steps` steps of SGD with momentum on one solver's rows, from the shared model; returns the solver's model.  `first`: the steps that it has
    made in the rounds before."""
    import torch
    own = [p.clone() for p in model.master]
    velocity = [torch.zeros_like(p) for p in own]
    n = tokens.shape[0]
    for h in range(steps):
        at = step_rows(first + h, batch, n, tokens.device)
        some, target = tokens[at], labels[at]
        count = (target >= 0).sum().clamp(min=1).float()
        row_weight = (loss_scale / count).expand(at.numel()).contiguous()
        _, grads = loss_and_gradients(ops, [p.to(model.dtype) for p in own], model.scale, some, target, row_weight)
        ops.clip_grads(grads, max_norm * loss_scale)
        for p, v, g in zip(own, velocity, grads):
            v.mul_(momentum).add_(g.float(), alpha=1.0 / loss_scale)
            p.add_(v, alpha=-rate)
    return own


def run_rounds(ops: TrainOps, model: TokenModel, tokens, labels, solvers: int, rounds: int, chunk_rows: int = 1024, steps: int = 16, batch: int = 1024,
               rate: float = 0.5, momentum: float = 0.9, max_norm: float = 1.0) -> Dict:
    """Rounds of local SGD; rows are chunks of chunk_rows, dealt to the solvers by `balance`; models are merged by samples."""
    import torch
    n = tokens.shape[0]
    chunks = [(i, min(n, i + chunk_rows)) for i in range(0, n, chunk_rows)]
    table = balance([b - a for a, b in chunks], solvers)
    rows = [torch.cat([torch.arange(a, b, device=tokens.device) for (a, b), k in zip(chunks, table) if k == s] or
                      [torch.empty(0, dtype=torch.long, device=tokens.device)]) for s in range(solvers)]
    loss_scale = 1024.0 if model.dtype == torch.float16 else 1.0
    losses, seconds = [evaluate(ops, model, tokens, labels)], 0.0
    for r in range(rounds):
        torch.cuda.synchronize()
        began = time.perf_counter()
        merged = [torch.zeros_like(p) for p in model.master]
        for own_rows in rows:
            if own_rows.numel() == 0:
                continue
            own = local_steps(ops, model, tokens[own_rows], labels[own_rows], steps, batch, rate, momentum, max_norm, loss_scale,
                              r * steps)
            for m, p in zip(merged, own):
                m.add_(p, alpha=own_rows.numel() / n)
        model.master = merged
        ops.sync()
        seconds += time.perf_counter() - began
        losses.append(evaluate(ops, model, tokens, labels))
    return {"losses": losses, "seconds": seconds, "rows_per_solver": [int(r.numel()) for r in rows]}


def synthetic_rows(rows: int, tokens: int, classes: int, seed: int, device: str):
    """Tokens with the popularity of words; a row's class follows from its token, with one row in ten at random and one in sixteen without."""
    import torch
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    u = torch.rand(rows, dtype=torch.float64, generator=gen, device=device)
    ids = ((tokens + 1.0) ** u).long().sub_(1).clamp_(0, tokens - 1)
    labels = ids * 2654435761 % classes
    odd = torch.rand(rows, generator=gen, device=device)
    labels = torch.where(odd < 0.1, torch.randint(0, classes, (rows,), generator=gen, device=device), labels)
    return ids.to(torch.int32), torch.where(odd > 1 - 1 / 16, -1, labels).to(torch.int32)


def main(argv=None) -> int:
    import torch
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rows", type=int, default=65536)
    ap.add_argument("--tokens", type=int, default=20000)
    ap.add_argument("--classes", type=int, default=5000)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--solvers", type=int, default=4)
    ap.add_argument("--rounds", type=int, default=8)
    ap.add_argument("--steps", type=int, default=16, help="H: local steps of a solver in a round")
    ap.add_argument("--batch", type=int, default=1024)
    ap.add_argument("--rate", type=float, default=0.5)
    ap.add_argument("--momentum", type=float, default=0.9)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--dtype", choices=TYPES, default="bfloat16")
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args(argv)
    device = "cuda:0"
    ops = TrainOps(device)
    ids, labels = synthetic_rows(args.rows, args.tokens, args.classes, args.seed, device)
    model = TokenModel(args.tokens, args.classes, args.width, getattr(torch, args.dtype), device, args.seed)
    out = run_rounds(ops, model, ids, labels, args.solvers, args.rounds, steps=args.steps, batch=args.batch, rate=args.rate, momentum=args.momentum,
                     max_norm=args.max_norm)
    for r, loss in enumerate(out["losses"]):
        print("round %2d: mean loss %.4f" % (r, loss), file=sys.stderr, flush=True)
    print(json.dumps(dict(vars(args), **out)))
    return 0


if __name__ == "__main__":
    sys.exit(main())
