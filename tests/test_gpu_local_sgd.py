"""Local SGD over categorical rows: the operators together, as a program uses them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
def test_loss_falls_over_rounds(dtype):
    import paper_1909_04885_amd as chicle
    from paper_1909_04885_amd.local_sgd import TokenModel, run_rounds, synthetic_rows
    ops = chicle.TrainOps("cuda:0")
    ids, labels = synthetic_rows(8000, 500, 300, 3, "cuda:0")
    model = TokenModel(500, 300, 64, dtype, "cuda:0")
    out = run_rounds(ops, model, ids, labels, solvers=3, rounds=3, chunk_rows=500, steps=12, batch=512)
    losses = out["losses"]
    assert sum(out["rows_per_solver"]) == 8000 and all(math.isfinite(v) for v in losses)
    # before training the scores are those of 64 products with a spread of one: about log(classes) + 1/2
    assert abs(losses[0] - (math.log(300) + 0.5)) < 0.5
    # nine rows of ten have the class that follows from their token: training gets below half of where it began
    assert losses[-1] < 0.5 * losses[0], losses


def test_one_step_against_automatic_differentiation():
    import paper_1909_04885_amd as chicle
    from paper_1909_04885_amd.local_sgd import TokenModel, loss_and_gradients, synthetic_rows
    ops = chicle.TrainOps("cuda:0")
    ids, labels = synthetic_rows(700, 200, 90, 5, "cuda:0")
    model = TokenModel(200, 90, 48, torch.float32, "cuda:0")
    weight = torch.rand(700, device="cuda")
    loss, grads = loss_and_gradients(ops, model.master, model.scale, ids, labels, weight)
    table, gamma, beta, w = [p.double().cpu().requires_grad_() for p in model.master]
    x = table[ids.long().cpu()] * model.scale
    mean = x.mean(1, keepdim=True)
    y = (x - mean) * ((x - mean).square().mean(1, keepdim=True) + 1e-5).rsqrt() * gamma + beta
    lse = torch.logsumexp(y @ w.t(), 1)
    has = labels.cpu() >= 0
    want = torch.where(has, lse - (y @ w.t())[torch.arange(700), labels.long().cpu().clamp(min=0)], 0.0)
    (want * weight.double().cpu()).sum().backward()
    # a chain of sums of at most 700 terms in 32 bits, each off by their number times 2^-24 at the most
    assert float((loss.double().cpu() - want.detach()).abs().max()) < 700 * 2.0 ** -24 * 10
    for got, p in zip(grads, (table, gamma, beta, w)):
        assert float((got.double().cpu() - p.grad).norm() / p.grad.norm()) < 700 * 2.0 ** -24
