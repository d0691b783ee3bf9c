"""Inputs of recurrences that remember for thousands of rows: what comes into a tile of 128 rows is still there after many of them, groups of 8 tiles and runs of
64, and a factor that is lost on the way shows."""
import torch

ROWS = 20000
LENGTHS = {"one": [ROWS], "some": [5, 4000, 0, 9000, 1, ROWS - 13006]}        # the latter begin and end inside tiles, groups and runs


def offsets_of(kind):
    at = [0]
    for x in LENGTHS[kind]:
        at.append(at[-1] + x)
    return at


def long_memory(kind, d, dtype):
    """f, u, offsets, h0, dy, dlast on the CPU.  Shares 1 - a from 2e-3 to 2e-6, by column, spread over a factor of e to both sides."""
    g = torch.Generator().manual_seed(d)
    f = (torch.linspace(6.0, 13.0, d) + torch.randn(ROWS, d, generator=g)).to(dtype)
    u, dy = (0.3 * torch.randn(ROWS, d, generator=g)).to(dtype), (0.01 * torch.randn(ROWS, d, generator=g)).to(dtype)
    k = len(LENGTHS[kind])
    h0, dlast = 1.0 + torch.rand(k, d, generator=g), 1.0 + torch.rand(k, d, generator=g)
    return f, u, offsets_of(kind), h0, dy, dlast
