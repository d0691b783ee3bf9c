"""Which rows the local SGD solvers train on, on the CPU: the steps themselves are left out."""
import pytest
import torch

import paper_1909_04885_amd.local_sgd as sgd


class Recorder:
    """Stands where the operators do: notes the tokens that it is asked for."""

    def __init__(self):
        self.tokens = []

    def embed(self, table, ids, scale=1.0):
        self.tokens.append(ids.clone())
        return torch.zeros(ids.shape[0], table.shape[1])

    def layer_norm(self, x, gamma, beta, eps=1e-5):
        return x, x[:, 0], x[:, 0]

    def softmax_loss(self, x, w, labels):
        return torch.zeros(x.shape[0]), torch.zeros(x.shape[0])

    def softmax_loss_grad(self, x, w, labels, weight):
        return torch.zeros(x.shape[0]), torch.zeros_like(x), torch.zeros_like(w)

    def layer_norm_grad(self, dy, x, gamma, mean, rstd):
        return dy, torch.zeros_like(gamma), torch.zeros_like(gamma)

    def embed_grad(self, ids, dout, n_rows, scale=1.0):
        return torch.zeros(n_rows, dout.shape[1])

    def clip_grads(self, grads, max_norm):
        return torch.zeros(())

    def sync(self):
        pass


@pytest.mark.parametrize("rows, rounds, steps, batch", [(1000, 5, 3, 32), (257, 3, 2, 16), (64, 2, 4, 16), (50, 2, 2, 64)])
def test_every_row_is_trained_on_as_often_as_the_others(monkeypatch, rows, rounds, steps, batch):
    monkeypatch.setattr(sgd, "evaluate", lambda *a, **k: 0.0)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)
    ops, solvers = Recorder(), 2
    model = sgd.TokenModel(rows, 5, 4, torch.float32, "cpu")
    out = sgd.run_rounds(ops, model, torch.arange(rows), torch.zeros(rows, dtype=torch.long), solvers, rounds, chunk_rows=8, steps=steps, batch=batch)
    assert sum(out["rows_per_solver"]) == rows
    times = torch.bincount(torch.cat(ops.tokens), minlength=rows)
    many = rounds * steps * batch
    # the rows of a solver are those of its chunks: each is met many / n times, rounded down or up
    assert int(times.sum()) == solvers * many
    owner = sgd.balance([min(8, rows - i) for i in range(0, rows, 8)], solvers)
    for s in range(solvers):
        own = torch.cat([torch.arange(i * 8, min(rows, i * 8 + 8)) for i, k in enumerate(owner) if k == s])
        n = own.numel()
        assert int(times[own].min()) >= many // n and int(times[own].max()) <= -(-many // n)
