"""Layers over sequences in local SGD: the operators together, as a program uses them."""
import math

import pytest
import torch

import sequence_reference as ref
from train_reference import U32

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ops():
    import paper_1909_04885_amd as chicle
    return chicle.TrainOps("cuda:0")


class Norm(torch.autograd.Function):
    """norm(r) gamma, whose gradient takes the values that were kept of r."""

    @staticmethod
    def forward(ctx, r, gamma, kept):
        rstd = ((r * r).mean(1, keepdim=True) + 1e-5).rsqrt()
        ctx.save_for_backward(kept, gamma, rstd)
        return r * rstd * gamma

    @staticmethod
    def backward(ctx, dy):
        kept, gamma, rstd = ctx.saved_tensors
        h, g = kept * rstd, dy * gamma
        return rstd * (g - h * (g * h).mean(1, keepdim=True)), (dy * h).sum(0), None


def values(x, d):
    return ref.unpack(x.values, x.scales, d).cpu() if isinstance(x, tuple) else x.double().cpu()


def by_differentiation(model, tokens, labels, weight, saved):
    """Loss and gradients in 64 bits, with what the package kept in 8 bits."""
    params = [p.double().cpu().requires_grad_() for p in model.master]
    t, d = tokens.long().cpu(), model.master[0].shape[1]
    r, h = params[0][t] * model.scale, None
    for k in range(model.layers + 1):
        y, kept = saved[k][0], values(saved[k][1], d)
        r = r if h is None else r + h
        u = Norm.apply(r, params[1 + 2 * k] if k < model.layers else params[-2], kept)
        if k == model.layers:
            break
        u = u + (values(y, d) - u).detach()
        a = torch.sigmoid(params[2 + 2 * k][t])
        rows, state = [], None
        for i in range(t.numel()):
            state = (1 - a[i]) * u[i] if i % model.length == 0 else a[i] * state + (1 - a[i]) * u[i]
            rows.append(state)
        h = torch.stack(rows)
    z = u @ params[-1].t()
    has = labels.cpu() >= 0
    loss = torch.where(has, torch.logsumexp(z, 1) - z[torch.arange(t.numel()), labels.long().cpu().clamp(min=0)], 0.0)
    (loss * weight.double().cpu()).sum().backward()
    return loss.detach(), [p.grad for p in params]


@pytest.mark.parametrize("keep8", [False, True])
@pytest.mark.parametrize("layers, length, rows", [(0, 7, 70), (1, 1, 40), (2, 40, 200), (3, 210, 420)])
def test_gradients_against_automatic_differentiation(ops, keep8, layers, length, rows):
    from paper_1909_04885_amd.local_sgd import SequenceModel, synthetic_sequences
    tokens, labels = synthetic_sequences(rows, length, 30, 20, 5, "cuda:0")
    model = SequenceModel(30, 20, 72, layers, length, F32, "cuda:0", 1, keep8)
    weight = torch.rand(rows, device="cuda") / rows
    loss, grads = model.loss_and_gradients(ops, model.master, tokens, labels, weight)
    _, saved = model.forward(ops, model.master, tokens, states=True)
    want_loss, want = by_differentiation(model, tokens, labels, weight, saved)
    # chains of at most 4 layers of sums of at most 420 terms in 32 bits, each off by their number times 2^-24 at the most
    tol = 4 * 420 * U32
    assert float((loss.double().cpu() - want_loss).abs().max()) < tol * 10
    assert len(grads) == len(model.master)
    for got, g, p in zip(grads, want, model.master):
        assert got.shape == p.shape
        assert float((got.double().cpu() - g).norm()) < tol * float(g.norm())
    ops.sync()


@pytest.mark.parametrize("keep8", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
def test_rows_one_by_one_give_what_whole_sequences_give(ops, dtype, keep8):
    """A program that answers goes on row by row from the layers' states."""
    from paper_1909_04885_amd.local_sgd import SequenceModel, synthetic_sequences
    sequences, length = 5, 37
    tokens, _ = synthetic_sequences(sequences * length, length, 50, 20, 2, "cuda:0")
    model = SequenceModel(50, 20, 64, 2, length, dtype, "cuda:0", 3, keep8)
    params = [p.to(dtype) for p in model.master]
    y = model.normed(ops, params, tokens).view(sequences, length, -1)
    states = model.first_states(sequences)
    stepped = torch.stack([model.step(ops, params, states, tokens.view(sequences, length)[:, t].contiguous()) for t in range(length)], 1)
    # The states differ by the order of sums alone; where a value lies at the border of two roundings (to the type, or to 8 bits, a step of 1/64 of the
    # largest of 32 values, of which none is above 6 times their root mean square here) it takes the other, and so may what follows from it
    off = (y.double() - stepped.double()).abs()
    if dtype == F32 and not keep8:
        assert float(off.max()) < 1e-5 * float(y.abs().max())
    else:
        assert float(off.square().mean().sqrt()) < (2 ** -6 if keep8 else 2 ** -8) * float(y.double().square().mean().sqrt())


@pytest.mark.parametrize("dtype, keep8", [(F32, False), (BF16, True), (F16, True)], ids=str)
def test_rounds_run(ops, dtype, keep8):
    from paper_1909_04885_amd.local_sgd import SequenceModel, run_rounds, synthetic_sequences
    ids, labels = synthetic_sequences(4000, 50, 200, 100, 3, "cuda:0")
    model = SequenceModel(200, 100, 64, 2, 50, dtype, "cuda:0", 0, keep8)
    out = run_rounds(ops, model, ids, labels, solvers=3, rounds=2, chunk_rows=500, steps=4, batch=250)
    assert sum(out["rows_per_solver"]) == 4000 and len(out["losses"]) == 3 and all(math.isfinite(v) for v in out["losses"])
    with pytest.raises(ValueError):
        run_rounds(ops, model, ids, labels, solvers=3, rounds=1, chunk_rows=512, steps=1, batch=250)


def test_the_command_runs(capsys):
    from paper_1909_04885_amd.local_sgd import main
    assert main("--rows 2048 --tokens 300 --classes 100 --width 40 --length 32 --layers 2 --keep8 --solvers 2 --rounds 1 --steps 2 --batch 256".split()) == 0
    assert '"keep8": true' in capsys.readouterr().out
