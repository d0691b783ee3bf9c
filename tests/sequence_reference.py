"""The operators of layers over sequences in 64 bits, on whatever device the inputs are, and the bounds the tests hold results to.

Bounds are worst cases of rounding, U32 = 2^-24 a rounding to 32 bits.  A gate's smaller share s is off by at most (10 + 2 |f|) U32 of itself: a power of two, a
reciprocal, each to a unit in the last place (two roundings), 1 + e and a product, each once, and what the exponent |f| log2(e) is off, which is rounded
once, as the factor is: (|f| log2(e)) 2 U32 ln(2) = 2 |f| U32.
"""
import torch

from train_reference import TINY, U, U32

GROUP, KEPT = 32, 32


def gate_off(f):
    return (10 + 2 * f.double().abs().clamp(max=104)) * U32


def pack(x):
    """(q, bytes) of rows whose values are given in any type, by whole numbers alone where it matters; not for infinities and NaN."""
    n, d = x.shape
    groups = -(-d // GROUP)
    wide = torch.zeros(n, groups * GROUP, dtype=torch.float64, device=x.device)
    wide[:, :d] = x
    wide = wide.view(n, groups, GROUP)
    top = wide.abs().amax(2)
    e = torch.full_like(top, -126.0)
    for k in range(-126, 123):                           # the least power of two that is enough
        e = torch.where(top > 127.0 * 2.0 ** k, torch.full_like(e, k + 1.0), e)
    q = torch.round(wide * torch.exp2(-e)[:, :, None])
    return q.view(n, groups * GROUP), (e + 127).to(torch.uint8)


def unpack(q, byte, d):
    step = torch.exp2(byte.double() - 127)
    return (q.double().view(*byte.shape, GROUP) * step[:, :, None]).view(q.shape)[:, :d]


def step_of(byte, d):
    """2^e for every column."""
    return torch.exp2(byte.double() - 127).repeat_interleave(GROUP, 1)[:, :d]


def rms_norm(x, gamma, residual, eps):
    dtype, d = x.dtype, x.shape[1]
    r = x if residual is None else (x.double() + residual.double()).to(dtype)
    wide, gamma = r.double(), gamma.double()
    rstd = 1.0 / torch.sqrt((wide * wide).mean(1) + eps)
    y = wide * rstd[:, None] * gamma
    off_rstd = rstd * (d / 8 + 40) * U32                 # a sum of squares, at least four of them side by side, in a tree
    off_y = y.abs() * (off_rstd / rstd)[:, None] + 4 * U32 * y.abs()       # (before it is rounded to the type)
    return {"r": r, "rstd": rstd, "y": y, "off_rstd": off_rstd, "off_y32": off_y, "off_y": off_y + U[dtype] * y.abs() + TINY[dtype]}


def rms_norm_grad(dy, r, gamma, rstd, dr):
    """r: values, of a type or in 64 bits."""
    dtype, (n, d) = dy.dtype, dy.shape
    dy, h, gamma, rstd = dy.double(), r.double() * rstd.double()[:, None], gamma.double(), rstd.double()[:, None]
    g = dy * gamma
    m = (g * h).mean(1, keepdim=True)
    off_m = (d / 8 + 44) * U32 * (g * h).abs().mean(1, keepdim=True)
    dx = rstd * (g - h * m)
    off = rstd * (h.abs() * off_m + 8 * U32 * (g.abs() + (h * m).abs()))
    if dr is not None:
        dx = dx + dr.double()
        off = off + 2 * U32 * dr.double().abs()
    dgamma = (dy * h).sum(0)
    off_gamma = (n + 8) * U32 * (dy * h).abs().sum(0)
    return {"dx": dx, "dgamma": dgamma, "off_dx": off + U[dtype] * dx.abs() + TINY[dtype],
            "off_dgamma": off_gamma + U[dtype] * dgamma.abs() + TINY[dtype]}


def gates(f):
    """(a, 1 - a, the smaller one), closed beyond +-104, in 64 bits."""
    f = f.double()
    a, c = torch.sigmoid(f), torch.sigmoid(-f)
    a, c = torch.where(f > 104, 1.0, torch.where(f < -104, 0.0, a)), torch.where(f > 104, 0.0, torch.where(f < -104, 1.0, c))
    return a, c, torch.minimum(a, c)


def share(a, x):
    """a x, nothing where a is 0."""
    return torch.where(a == 0, torch.zeros_like(x), a * x)


def scan(f, u, offsets, h0):
    """f, u [n, d] in any type, offsets a list: h, the states that enter rows, those after the sequences, and how far h may be off before it is rounded."""
    n, d = f.shape
    a, c, s = gates(f)
    gate = gate_off(f)
    u = u.double()
    h, before, off = torch.zeros_like(a), torch.zeros_like(a), torch.zeros_like(a)
    k = len(offsets) - 1
    last = torch.zeros(k, d, dtype=torch.float64, device=f.device) if h0 is None else h0.double().clone()
    off_last = torch.zeros_like(last)
    off_before = torch.zeros_like(a)
    for j in range(k):
        x, e = last[j].clone(), torch.zeros_like(last[j])
        for t in range(offsets[j], offsets[j + 1]):
            before[t], off_before[t] = x, e
            parts = share(a[t], x).abs() + share(c[t], u[t]).abs()
            seen = share(s[t], x).abs() + share(s[t], u[t]).abs()
            e = share(a[t], e) + 2 * (gate[t] * seen + 2 * U32 * parts)       # twice: rows are also carried as a product of shares and a sum
            x = share(a[t], x) + share(c[t], u[t])
            h[t], off[t] = x, e
        last[j], off_last[j] = x, e
    return {"h": h, "off": off, "before": before, "off_before": off_before, "last": last, "off_last": off_last}


def scan_grad(f, u, offsets, h0, dy, dlast):
    dtype = f.dtype
    r = scan(f, u, offsets, h0)
    a, c, s = gates(f)
    gate = gate_off(f)
    u, dy = u.double(), dy.double()
    k, d = len(offsets) - 1, f.shape[1]
    g, off = torch.zeros_like(a), torch.zeros_like(a)
    dh0 = torch.zeros(k, d, dtype=torch.float64, device=f.device) if dlast is None else dlast.double().clone()
    off_dh0 = torch.zeros_like(dh0)
    for j in range(k):
        x, e = dh0[j].clone(), torch.zeros_like(dh0[j])
        for t in range(offsets[j + 1] - 1, offsets[j] - 1, -1):
            x, e = x + dy[t], e + 2 * U32 * (x + dy[t]).abs() + 2 * U32 * x.abs()
            g[t], off[t] = x, e
            e = share(a[t], e) + 2 * (gate[t] * share(s[t], x).abs() + 2 * U32 * share(a[t], x).abs())
            x = share(a[t], x)
        dh0[j], off_dh0[j] = x, e
    wide = r["before"] - u
    slope = a * c
    df, du = share(slope, g * wide), share(c, g)
    off_df = share(slope, off * wide.abs() + g.abs() * (r["off_before"] + 2 * U32 * wide.abs())) + (2 * gate + 8 * U32) * df.abs()
    off_du = share(c, off) + 2 * gate * share(s, g).abs() + 2 * U32 * du.abs()
    return {"df": df, "du": du, "dh0": dh0, "off_df": off_df + U[dtype] * df.abs() + TINY[dtype], "off_du": off_du + U[dtype] * du.abs() + TINY[dtype],
            "off_dh0": off_dh0 + 2 * U32 * dh0.abs() + TINY[torch.float32]}
