"""The operators of a training step whose speed is followed, in the plain form that says what they compute and as calls of the package.

They belong to local SGD over categorical data (the second application beside CoCoA): rows of a table are looked up by
token, normalised, scored against many classes with the softmax loss, and the gradients of a step are clipped by their
common norm before they are applied.

  loss        softmax cross entropy of rows x [n, d] against w [classes, d]; a negative label: the row has none
  loss_grad   the same with the gradients of sum_i weight_i loss_i by x and w
  embed       out[i] = scale * table[id_i]
  embed_grad  dtable[v] = scale * sum over the i with id_i = v of dout[i]
  norm        layer norm with weight and bias
  norm_grad   its gradients by the input, the weight and the bias
  clip        the norm of many tensors together, and the tensors times min(1, max_norm / (norm + 1e-6))
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
MOST_CLASSES_ROWS = 8192 * 128000      # logits that the plain form holds at once: 4 GB in 32 bits


def _case(op, name=None, **fields):
    return dict({"op": op}, **({} if name is None else {"name": name}), **fields)


def listed():
    return [
        # one row scored against a vocabulary while a model answers: the weights are read once, latency counts
        _case("loss", "loss_one", n=1, d=1024, classes=32000, dtype="bf16", extra=0),
        # a small local solver's step in the framework's own type, sizes that divide by nothing
        _case("loss_grad", "loss_grad_small", n=333, d=250, classes=20000, dtype="f32", extra=6),
        # an ordinary training step, a number of classes that is no multiple of anything
        _case("loss_grad", "loss_grad", n=4096, d=1024, classes=50021, dtype="bf16", extra=0),
        # a long batch against a large vocabulary
        _case("loss_grad", "loss_grad_large", n=8192, d=2048, classes=128000, dtype="bf16", extra=0),
        # the tokens of a batch of prompts
        _case("embed", "embed_prompts", n=16001, d=2048, classes=128000, dtype="f16", wide_ids=True),
        # a sparse data set's columns, 200 thousand of them, in the framework's own type
        _case("embed_grad", "embed_grad", n=30011, d=256, classes=200000, dtype="f32", wide_ids=False),
        # the step of a large vocabulary: popular tokens come thousands of times
        _case("embed_grad", "embed_grad_large", n=131072, d=2048, classes=128000, dtype="bf16", wide_ids=True),
        # one row while a model answers: latency
        _case("norm", "norm_one", n=1, d=4096, dtype="bf16", extra=0),
        # odd rows of a wider buffer
        _case("norm_grad", "norm_grad", n=9001, d=1537, dtype="f32", extra=3),
        # a long batch of wide rows
        _case("norm_grad", "norm_grad_large", n=65536, d=4096, dtype="bf16", extra=0),
        # the gradients of a small model: many small tensors
        _case("clip", "clip_small", layers=8, d=250, classes=2000, dtype="f32", clipped=True),
        # the gradients of a large one
        _case("clip", "clip_large", layers=5, d=4096, classes=128000, dtype="bf16", clipped=True),
    ]


def _log_uniform(rng, lo, hi):
    size = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return size - (size == 3 * 1024)                         # (a size that is not used here)


def draw(rng):
    op = rng.choice(["loss", "loss_grad", "loss_grad", "embed", "embed_grad", "embed_grad", "norm", "norm_grad", "clip"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op in ("loss", "loss_grad"):
        while True:
            n, d, c = _log_uniform(rng, 1, 8192), _log_uniform(rng, 48, 4096), _log_uniform(rng, 1000, 256000)
            if rng.random() < 0.5:
                d = max(64, d // 128 * 128 + 64)
            # 32-bit products cost several times as much
            if n * c <= MOST_CLASSES_ROWS and n * c * d * (8 if dtype == "f32" else 1) <= 8192 * 2048 * 128000:
                return _case(op, n=n, d=d, classes=c, dtype=dtype, extra=rng.choice([0, 0, 5, 8]))
    if op in ("embed", "embed_grad"):
        while True:
            n, d, c = _log_uniform(rng, 1, 200000), _log_uniform(rng, 16, 4096), _log_uniform(rng, 1000, 1000000)
            size = 4 if dtype == "f32" else 2
            if (n + c) * d * size <= (131072 + 128000) * 2048 * 2:
                return _case(op, n=n, d=d, classes=c, dtype=dtype, wide_ids=rng.random() < 0.5)
    if op in ("norm", "norm_grad"):
        while True:
            n, d = _log_uniform(rng, 1, 200000), _log_uniform(rng, 16, 16384)
            if n * d * (4 if dtype == "f32" else 2) <= 65536 * 4096 * 2:
                return _case(op, n=n, d=d, dtype=dtype, extra=rng.choice([0, 0, 3, 8]))
    while True:
        layers, d, c = rng.randint(0, 8), _log_uniform(rng, 16, 4096), _log_uniform(rng, 500, 256000)
        if (c * d + 9 * layers * d * d) * (4 if dtype == "f32" else 2) <= (128000 * 4096 + 45 * 4096 * 4096) * 2:
            return _case(op, layers=layers, d=d, classes=c, dtype=dtype, clipped=rng.random() < 0.75)


def _zipf_cdf(classes):
    p = torch.arange(1, classes + 1, dtype=torch.float64, device=DEVICE).pow(-1.1).cumsum(0)
    return p / p[-1]


def _zipf(gen, n, classes):
    """Tokens with the popularity of words: the r-th most frequent has a probability in proportion to r^-1.1."""
    u = torch.rand(n, dtype=torch.float64, device=DEVICE, generator=gen)
    return torch.searchsorted(_zipf_cdf(classes), u).clamp_(max=classes - 1)


def _normal(gen, shape, dtype, spread=1.0, mean=0.0):
    return torch.empty(shape, dtype=TYPE[dtype], device=DEVICE).normal_(mean, spread, generator=gen)


def _rows(gen, n, d, extra, dtype, spread=1.0):
    """n rows of d in a buffer whose rows are `extra` values longer."""
    return _normal(gen, (n, d + extra), dtype, spread)[:, :d]


def _grad_shapes(case):
    d, shapes = case["d"], [(case["classes"], case["d"])]
    for _ in range(case["layers"]):
        shapes += [(d, d), (d, 4 * d), (4 * d, d), (4 * d,), (d,), (d,)]
    return shapes


def _ops():
    import paper_1909_04885_amd as chicle
    return chicle.TrainOps(DEVICE)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    s = dict(case, ops=_ops() if own else None)
    op, dtype = case["op"], case["dtype"]
    if op in ("loss", "loss_grad"):
        n, d, c = case["n"], case["d"], case["classes"]
        s["x"] = _rows(gen, n, d, case["extra"], dtype)
        s["w"] = _rows(gen, c, d, case["extra"], dtype, 1.5 / math.sqrt(d))
        labels = _zipf(gen, n, c).to(torch.int32)
        if n > 1:                                            # one row in sixteen has no label
            labels[torch.rand(n, device=DEVICE, generator=gen) < 1 / 16] = -1
            labels[:1] = 0
        s["labels"] = labels
        # the mean over the rows with a label; in 16 bits with few exponents the loss comes scaled, so that gradients do not vanish
        s["weight"] = (labels >= 0).float() * (4096.0 if dtype == "f16" else 1.0) / (labels >= 0).sum()
    elif op in ("embed", "embed_grad"):
        n, d, c = case["n"], case["d"], case["classes"]
        s["ids"] = _zipf(gen, n, c).to(torch.int64 if case["wide_ids"] else torch.int32)
        s["scale"] = math.sqrt(d)
        if op == "embed":
            s["table"] = _normal(gen, (c, d), dtype, 1 / math.sqrt(d))
        else:
            s["dout"] = _normal(gen, (n, d), dtype, 1 / math.sqrt(n))
    elif op in ("norm", "norm_grad"):
        n, d = case["n"], case["d"]
        s["x"] = _rows(gen, n, d, case["extra"], dtype, 2.0)
        s["gamma"] = _normal(gen, (d,), dtype, 0.1, 1.0)
        s["beta"] = _normal(gen, (d,), dtype, 0.1)
        if op == "norm_grad":                                # a step has the forward pass's statistics in hand
            s["dy"] = _rows(gen, n, d, case["extra"], dtype, 1 / math.sqrt(n))
            s["mean"], s["rstd"] = _moments(s["x"])
    else:
        s["grads"] = [_normal(gen, shape, dtype, 1e-3) for shape in _grad_shapes(case)]
        s["out"] = [torch.empty_like(g) for g in s["grads"]]
        s["max_norm"] = 0.37 * 1e-3 * math.sqrt(sum(g.numel() for g in s["grads"])) if case["clipped"] else 1e4
    return s


def _moments(x):
    x = x.float()
    mean = x.mean(1)
    return mean, ((x - mean[:, None]).square().mean(1) + EPS).rsqrt()


def run(s):
    op = s["op"]
    if own:
        ops = s["ops"]
        if op == "loss":
            return ops.softmax_loss(s["x"], s["w"], s["labels"])
        if op == "loss_grad":
            return ops.softmax_loss_grad(s["x"], s["w"], s["labels"], s["weight"])
        if op == "embed":
            return ops.embed(s["table"], s["ids"], s["scale"])
        if op == "embed_grad":
            return ops.embed_grad(s["ids"], s["dout"], s["classes"], s["scale"])
        if op == "norm":
            return ops.layer_norm(s["x"], s["gamma"], s["beta"], EPS)
        if op == "norm_grad":
            return ops.layer_norm_grad(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"])
        return ops.clip_grads(s["grads"], s["max_norm"], s["out"]), s["out"]
    if op in ("loss", "loss_grad"):
        x, w, labels = s["x"].float(), s["w"].float(), s["labels"].long()
        logits = x @ w.t()
        top = logits.amax(1, keepdim=True)
        lse = (logits - top).exp_().sum(1).log() + top[:, 0]
        has = labels >= 0
        picked = logits.gather(1, labels.clamp(min=0)[:, None])[:, 0]
        loss = torch.where(has, lse - picked, torch.zeros_like(lse))
        if op == "loss":
            return loss, lse
        p = logits.sub_(lse[:, None]).exp_()
        at = torch.arange(p.shape[0], device=p.device)
        p[at, labels.clamp(min=0)] -= 1.0
        p *= torch.where(has, s["weight"], torch.zeros_like(lse))[:, None]
        return loss, (p @ w).to(s["x"].dtype), (p.t() @ x).to(s["w"].dtype)
    if op == "embed":
        return (s["table"][s["ids"].long()].float() * s["scale"]).to(s["table"].dtype)
    if op == "embed_grad":
        dout = s["dout"]
        total = torch.zeros(s["classes"], dout.shape[1], dtype=torch.float32, device=dout.device)
        total.index_add_(0, s["ids"].long(), dout.float())
        return (total * s["scale"]).to(dout.dtype)
    if op == "norm":
        mean, rstd = _moments(s["x"])
        y = (s["x"].float() - mean[:, None]) * rstd[:, None] * s["gamma"].float() + s["beta"].float()
        return y.to(s["x"].dtype), mean, rstd
    if op == "norm_grad":
        dy, rstd, dtype = s["dy"].float(), s["rstd"][:, None], s["x"].dtype
        xhat = (s["x"].float() - s["mean"][:, None]) * rstd
        g = dy * s["gamma"].float()
        dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        return dx.to(dtype), (dy * xhat).sum(0).to(dtype), dy.sum(0).to(dtype)
    squares = torch.stack([g.float().square().sum() for g in s["grads"]])
    norm = squares.sum().sqrt()
    factor = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    return norm, [(g.float() * factor).to(g.dtype) for g in s["grads"]]


def work(case):
    op, size = case["op"], 4 if case["dtype"] == "f32" else 2
    d = case["d"]
    if op in ("loss", "loss_grad"):
        n, c = case["n"], case["classes"]
        once = (n + c) * d * size
        if op == "loss":
            return {"bytes": once + 12 * n, "flops": 2 * n * c * d}
        return {"bytes": 2 * once + 12 * n, "flops": 6 * n * c * d}
    if op in ("embed", "embed_grad"):
        n, c = case["n"], case["classes"]
        ids = n * (8 if case["wide_ids"] else 4)
        if op == "embed_grad":
            return {"bytes": ids + (n + c) * d * size, "flops": n * d}
        distinct = sum(-math.expm1(n * math.log1p(-p)) if p < 1 else 1.0 for p in _zipf_probabilities(c))
        return {"bytes": int(ids + (n + distinct) * d * size), "flops": n * d}
    if op == "norm":
        return {"bytes": (2 * case["n"] * d + 2 * d) * size + 8 * case["n"], "flops": 8 * case["n"] * d}
    if op == "norm_grad":
        return {"bytes": (3 * case["n"] * d + 3 * d) * size + 8 * case["n"], "flops": 15 * case["n"] * d}
    total = sum(math.prod(shape) for shape in _grad_shapes(case))
    return {"bytes": 2 * total * size + 4, "flops": 3 * total}


def _zipf_probabilities(classes):
    p = [r ** -1.1 for r in range(1, classes + 1)]
    total = sum(p)
    return [x / total for x in p]


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    op = case["op"]
    if op in ("loss", "loss_grad"):
        if 6 * case["n"] * case["d"] * case["classes"] > 2e13 or case["n"] * case["classes"] > 1.1 * MOST_CLASSES_ROWS:
            return None
        x, w = s["x"].double(), s["w"].double()
        z = torch.mm(x, w.t().contiguous())
        rows = torch.arange(case["n"], device=DEVICE)
        labels = s["labels"].long()
        valid = (labels >= 0).double()
        target = labels * (labels >= 0)
        lse = torch.logsumexp(z, dim=1)
        loss = valid * (lse - z[rows, target])
        if op == "loss":
            return loss, lse
        z = torch.exp(z - lse.unsqueeze(1))
        z.index_put_((rows, target), torch.full((1,), -1.0, dtype=torch.float64, device=DEVICE).expand(case["n"]), accumulate=True)
        z.mul_((valid * s["weight"].double()).unsqueeze(1))
        return loss, torch.mm(z, w), torch.mm(z.t().contiguous(), x)
    if op == "embed":
        return torch.nn.functional.embedding(s["ids"].long(), s["table"]).double().mul_(s["scale"])
    if op == "embed_grad":
        ids, order = torch.sort(s["ids"].long(), stable=True)
        out = torch.zeros(case["classes"], case["d"], dtype=torch.float64, device=DEVICE)
        step = max(1, (1 << 26) // case["d"])
        for i in range(0, case["n"], step):
            out.index_put_((ids[i:i + step],), s["dout"][order[i:i + step]].double(), accumulate=True)
        return out.mul_(s["scale"])
    x = s.get("x")
    if op == "norm":
        var, mean = torch.var_mean(x.double(), dim=1, correction=0)
        rstd = 1.0 / torch.sqrt(var + EPS)
        return (x.double() - mean.unsqueeze(1)).mul_(rstd.unsqueeze(1)).mul_(s["gamma"].double()).add_(s["beta"].double()), mean, rstd
    if op == "norm_grad":
        d, dy, gamma = case["d"], s["dy"].double(), s["gamma"].double()
        h = (x.double() - s["mean"].double().unsqueeze(1)).mul_(s["rstd"].double().unsqueeze(1))
        weighted = dy * gamma
        a, b = weighted.sum(1, keepdim=True) / d, (weighted * h).sum(1, keepdim=True) / d
        dgamma, dbeta = (dy * h).sum(0), dy.sum(0)
        dx = weighted.sub_(a).sub_(h.mul_(b)).mul_(s["rstd"].double().unsqueeze(1))
        return dx, dgamma, dbeta
    norm = math.sqrt(sum(float(torch.linalg.vector_norm(g.reshape(-1), dtype=torch.float64)) ** 2 for g in s["grads"]))
    factor = min(1.0, s["max_norm"] / (norm + 1e-6))
    return norm, [g.double() * factor for g in s["grads"]]
