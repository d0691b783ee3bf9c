"""The training operators' definitions in 64 bits on whatever device the inputs are, and the bounds the tests hold results to.

Bounds are worst cases of rounding: a sum of k products in 32 bits, added up in any order of depth t, is off by at most
(t + 2) 2^-24 times the sum of the products' magnitudes; a result of type T is rounded once more, by at most its unit
round-off U[T] of itself, and by half the smallest subnormal where it is that small.
"""
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
U32 = 2.0 ** -24


def within(got, want, bound, what=""):
    got, want = got.double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), "of", bad.numel(), "largest", float(off.nan_to_num(float("inf")).max()))


def softmax_loss(x, w, labels, weight=None):
    """loss, lse, dx, dw and bounds of their errors (a dict) for inputs of any type; rows with a label that is negative count nowhere."""
    dtype = x.dtype
    n, d = x.shape
    classes = w.shape[0]
    has = labels >= 0
    x = torch.where(has[:, None], x.double(), torch.zeros((), dtype=torch.float64, device=x.device))
    w = w.double()
    z = x @ w.t().contiguous()
    size = x.abs() @ w.abs().t().contiguous()
    lse = torch.logsumexp(z, 1)
    at = torch.arange(n, device=x.device)
    target = labels.long().clamp(min=0)
    loss = torch.where(has, lse - z[at, target], torch.zeros_like(lse))
    depth = d + 8                                        # (products of one sum, planes of a 32-bit operand among them six times)
    off_z = 6 * depth * U32 * size if dtype == torch.float32 else depth * U32 * size
    # exponentials of differences, their sums over all classes, the logarithm
    off_lse = off_z.max(1).values + (classes / 16 + 64) * U32 + 8 * U32 * z.abs().amax(1)
    out = {"loss": loss, "lse": lse, "has": has, "off_lse": off_lse, "off_loss": off_lse + off_z[at, target] + 4 * U32 * (lse.abs() + z[at, target].abs())}
    if weight is None:
        return out
    weight = torch.where(has, weight.double(), torch.zeros_like(lse))
    p = torch.exp(z - lse[:, None])
    g = p.clone()
    g[at, target] -= 1.0
    g *= weight[:, None]
    wide = weight.abs()[:, None]
    # of G: what its exponential is off by, its own rounding, and in half precision what is below the smallest subnormal after scaling
    off_g = wide * p * (2 * (off_z + off_lse[:, None]) + 8 * U32 * (z - lse[:, None]).abs().clamp(max=200.0)) + 2 * U[dtype] * g.abs() + 4 * U32 * wide
    if dtype == torch.float16:
        off_g = off_g + 2.0 ** -37 * wide.max()
    for name, product, mass, off, k in (("dx", g @ w, g.abs() @ w.abs(), off_g @ w.abs(), classes),
                                        ("dw", g.t().contiguous() @ x, g.abs().t().contiguous() @ x.abs(), off_g.t().contiguous() @ x.abs(), n)):
        out[name] = product
        out["off_" + name] = off + 6 * (k + 64) * U32 * mass + U[dtype] * product.abs() + TINY[dtype]
    return out


def layer_norm(x, gamma, beta, eps):
    dtype, d = x.dtype, x.shape[1]
    x, gamma, beta = x.double(), gamma.double(), beta.double()
    mean = x.mean(1)
    c = x - mean[:, None]
    var = (c * c).mean(1)
    rstd = (var + eps).rsqrt()
    y = c * rstd[:, None] * gamma + beta
    depth = d / 8 + 32
    off_mean = (depth + 2) * U32 * x.abs().mean(1)
    # the variance is off by its own sum and by the square of what the mean is off
    off_rstd = rstd * ((depth + 8) * U32 + 0.5 * rstd * rstd * (off_mean ** 2 + 2 * U32 * x.abs().amax(1) * c.abs().mean(1)))
    off_c = off_mean[:, None] + 2 * U32 * x.abs()
    off_y = (off_c * rstd[:, None] + c.abs() * off_rstd[:, None]) * gamma.abs() + 8 * U32 * (c.abs() * rstd[:, None] * gamma.abs() + beta.abs()) + \
        U[dtype] * y.abs() + TINY[dtype]
    return {"y": y, "mean": mean, "rstd": rstd, "off_y": off_y, "off_mean": off_mean, "off_rstd": off_rstd}


def layer_norm_grad(dy, x, gamma, mean, rstd):
    dtype, (n, d) = x.dtype, x.shape
    dy, x, gamma, mean, rstd = dy.double(), x.double(), gamma.double(), mean.double()[:, None], rstd.double()[:, None]
    h = (x - mean) * rstd
    off_h = 2 * U32 * (x.abs() + mean.abs()) * rstd + 2 * U32 * h.abs()
    g = dy * gamma
    a, b = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    depth = d / 8 + 40
    off_a = depth * U32 * g.abs().mean(1, keepdim=True)
    off_b = depth * U32 * (g * h).abs().mean(1, keepdim=True) + (g.abs() * off_h).mean(1, keepdim=True)
    dx = rstd * (g - a - h * b)
    off_dx = rstd * (off_a + h.abs() * off_b + off_h * b.abs() + 8 * U32 * (g.abs() + a.abs() + (h * b).abs())) + U[dtype] * dx.abs() + TINY[dtype]
    dgamma, dbeta = (dy * h).sum(0), dy.sum(0)
    off_dgamma = (n + 8) * U32 * (dy * h).abs().sum(0) + (dy.abs() * off_h).sum(0) + U[dtype] * dgamma.abs() + TINY[dtype]
    off_dbeta = (n + 8) * U32 * dy.abs().sum(0) + U[dtype] * dbeta.abs() + TINY[dtype]
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta, "off_dx": off_dx, "off_dgamma": off_dgamma, "off_dbeta": off_dbeta}


def embed_grad(ids, dout, n_rows, scale, into=None):
    """The sums and their bounds; `into` is what they are added to."""
    dtype, d = dout.dtype, dout.shape[1]
    keep = (ids >= 0) & (ids < n_rows)
    total = torch.zeros(n_rows, d, dtype=torch.float64, device=dout.device)
    mass = torch.zeros_like(total)
    total.index_add_(0, ids[keep].long(), dout[keep].double() * scale)
    mass.index_add_(0, ids[keep].long(), dout[keep].double().abs() * abs(scale))
    count = torch.bincount(ids[keep].long(), minlength=n_rows).double()[:, None]
    off = (count + 4) * U32 * mass
    if into is not None:
        total = total + into.double()
        off = off + 2 * U32 * total.abs()
    touched = count[:, 0] > 0
    off = off + torch.where(touched[:, None], U[dtype] * total.abs() + TINY[dtype], torch.zeros_like(total))
    return total, off
