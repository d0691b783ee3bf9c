"""The softmax loss's gradients against bounds that hold row by row and class by class: what 32-bit sums of these very terms are off by at the most,
what is held in fewer bits on the way, and the rounding of the results.

A sum of k products in 32 bits is off by at most (k + 8) 2^-24 times the sum of the products' magnitudes.  G = weight (softmax - onehot) is held to
twice the bits of a 16-bit type, an error of HELD of itself.
"""
import math

import pytest
import torch

from train_reference import TINY, U, U32, within

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAME = {F32: "f32", BF16: "bf16", F16: "f16"}
HELD = {F32: 0.0, BF16: U[BF16] ** 2, F16: U[F16] ** 2}


@pytest.fixture(scope="module")
def ops():
    import paper_1909_04885_amd as chicle
    return chicle.TrainOps("cuda:0")


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, n, d, dtype, spread=1.0, extra=0, shift=0):
    return (torch.randn(n, shift + d + extra, generator=g, device="cuda") * spread).to(dtype)[:, shift:shift + d]


def check_gradients(ops, x, w, labels, weight):
    dtype, (n, d), classes = x.dtype, x.shape, w.shape[0]
    loss, dx, dw = ops.softmax_loss_grad(x, w, labels, weight)
    has = labels >= 0
    xd, wd = torch.where(has[:, None], x.double(), torch.zeros((), dtype=torch.float64, device="cuda")), w.double()
    z, size = xd @ wd.t().contiguous(), xd.abs() @ wd.abs().t().contiguous()
    lse = torch.logsumexp(z, 1)
    rows, target = torch.arange(n, device="cuda"), labels.long().clamp(min=0)
    off_z = (d + 8) * U32 * size
    del size
    off_lse = off_z.amax(1) + (classes / 16 + 64) * U32 + 8 * U32 * z.abs().amax(1)
    want = torch.where(has, lse - z[rows, target], torch.zeros_like(lse))
    within(loss, want, torch.where(has, off_lse + off_z[rows, target] + 4 * U32 * (lse.abs() + z[rows, target].abs()), torch.zeros_like(lse)), "loss")
    wide = torch.where(has, weight.double(), torch.zeros_like(lse))[:, None]
    p = torch.exp(z - lse[:, None])
    off_g = wide.abs() * (p * (2 * (off_z + off_lse[:, None]) + 8 * U32 * (z - lse[:, None]).abs().clamp(max=200.0)) + 4 * U32)
    del off_z, z
    p[rows, target] -= 1.0
    g = p * wide
    del p
    off_g += HELD[dtype] * g.abs()
    if dtype == F16:                                     # what lies below half precision's smallest value, of the largest weight's 2^14
        off_g += 2.0 ** -38 * wide.abs().max() * (wide != 0)
    for name, got, left, right, off, k in (("dx", dx, g, wd, off_g, classes), ("dw", dw, g.t().contiguous(), xd, off_g.t().contiguous(), n)):
        exact = left @ right
        bound = off @ right.abs() + (k + 64) * U32 * (left.abs() @ right.abs()) + U[dtype] * exact.abs() + TINY[dtype]
        within(got, exact, bound, name)
    ops.sync()
    return dx, dw


@pytest.mark.parametrize("n, classes", [(3, 400), (40, 300), (256, 600), (4100, 3100)])
@pytest.mark.parametrize("weights", ["one", "uneven"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=NAME.get)
def test_what_classes_have_in_common_drops_out(ops, dtype, weights, n, classes):
    """Rows of G add up to zero, so what all classes hold in a column gives that column of dx nothing: errors of G must not add up there.  The
    columns of the common mean are such in which x is zero, so that the logits do not carry it; and x has a mean where w is zero."""
    print("\ncase common mean", NAME[dtype], weights, n, classes, flush=True)
    g = gen(n)
    d = 144
    x, w = normal(g, n, d, dtype), normal(g, classes, d, dtype, 1.5 / math.sqrt(64))
    x[:, 64:128] = 0.0
    w[:, 64:128] = (4 * torch.randn(64, generator=g, device="cuda")).to(dtype)
    x[:, 128:] = (4 * torch.randn(16, generator=g, device="cuda")).to(dtype)
    w[:, 128:] = 0.0
    labels = (x.float() @ w.float().t()).argmax(1)
    labels[n // 2:] = torch.randint(-1, classes, (n - n // 2,), generator=g, device="cuda")
    weight = torch.full((n,), 1.0 / n, device="cuda") if weights == "one" else torch.rand(n, generator=g, device="cuda") * 8
    check_gradients(ops, x, w, labels, weight)


@pytest.mark.parametrize("value", [1e9, 1e20, 1e35])
@pytest.mark.parametrize("n", [5, 40, 300, 4100])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=NAME.get)
def test_the_weight_of_a_row_without_a_label_counts_nowhere(ops, dtype, n, value):
    """Finite and larger than all others, and that of a row whose label is past the end too."""
    import paper_1909_04885_amd as chicle
    g = gen(n)
    x, w = normal(g, n, 96, dtype), normal(g, 3100, 96, dtype, 0.15)
    labels = torch.randint(0, 3100, (n,), generator=g, device="cuda", dtype=torch.int32)
    weight = torch.rand(n, generator=g, device="cuda") + 0.5
    labels[1], weight[1] = -1, value
    want = check_gradients(ops, x, w, labels, weight)
    labels[1] = 3100
    got = ops.softmax_loss_grad(x, w, labels, weight)[1:]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(chicle.ChicleError, match="label"):
        ops.sync()


@pytest.mark.parametrize("n, d, classes", [(50000, 72, 12000), (20000, 16, 30000), (16384, 200, 32700)])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=NAME.get)
def test_pieces_of_the_classes_share_the_rows_gradient(ops, dtype, n, d, classes):
    """Several pieces, each added to what the ones before left: in large tiles, in middle tiles whose sums are divided, in large ones that are."""
    print("\ncase pieces", NAME[dtype], n, d, classes, flush=True)
    g = gen(n)
    x, w = normal(g, n, d, dtype), normal(g, classes, d, dtype, 1.0 / math.sqrt(d))
    labels = torch.randint(-1, classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    check_gradients(ops, x, w, labels, torch.rand(n, generator=g, device="cuda"))


@pytest.mark.parametrize("n, d, classes, extra", [(4100, 1030, 33001, 3), (4096, 1024, 33000, 0)])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=NAME.get)
def test_large_tiles_of_long_sums(ops, dtype, n, d, classes, extra):
    """Tiles of 256 x 256 in every product, sixteen slices of k and more, dx's sum divided; once with remainders on all sides, once with w read as
    it lies."""
    print("\ncase large tiles", NAME[dtype], n, d, classes, flush=True)
    g = gen(classes)
    x, w = normal(g, n, d, dtype, 1.0, extra), normal(g, classes, d, dtype, 1.0 / math.sqrt(d), extra)
    labels = torch.randint(-1, classes, (n,), generator=g, device="cuda")
    labels[-40:] = torch.arange(classes - 40, classes, device="cuda")
    first = check_gradients(ops, x, w, labels, torch.rand(n, generator=g, device="cuda"))
    del first
    weight = torch.full((n,), 1.0, device="cuda")
    a, b = ops.softmax_loss_grad(x, w, labels, weight), ops.softmax_loss_grad(x, w, labels, weight)
    assert all(torch.equal(s, t) for s, t in zip(a, b))   # whatever the timing


@pytest.mark.parametrize("n", [3, 200, 5000])
@pytest.mark.parametrize("scale", [2.0 ** -6, 1.0, 4096.0])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=NAME.get)
def test_weights_of_many_powers_of_two_in_one_call(ops, dtype, scale, n):
    """Every row of dx against its own weight, down to 2^-18 of the largest."""
    g = gen(n + 1)
    x, w = normal(g, n, 64, dtype), normal(g, 3100, 64, dtype, 0.2)
    labels = torch.randint(0, 3100, (n,), generator=g, device="cuda", dtype=torch.int32)
    weight = scale * (1 + torch.rand(n, generator=g, device="cuda")) * 2.0 ** -torch.randint(0, 18, (n,), generator=g, device="cuda").float()
    check_gradients(ops, x, w, labels, weight)


@pytest.mark.parametrize("n, d, classes, extra, shift", [
    (1, 64, 1, 0, 0), (1, 200, 1000, 0, 0), (3, 65, 257, 1, 0), (17, 100, 700, 3, 5), (24, 1030, 900, 2, 0), (65, 192, 1000, 8, 0), (100, 250, 2000, 6, 0),
    (128, 512, 1024, 0, 0), (129, 320, 777, 0, 3), (300, 2050, 700, 0, 0), (600, 130, 3001, 0, 0), (2500, 64, 500, 0, 0)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=NAME.get)
def test_gradients_of_all_sizes(ops, dtype, n, d, classes, extra, shift):
    print("\ncase all sizes", NAME[dtype], n, d, classes, extra, shift, flush=True)
    g = gen(n * d + classes)
    x, w = normal(g, n, d, dtype, 1.0, extra, shift), normal(g, classes, d, dtype, 2.0 / math.sqrt(d), extra, shift)
    labels = torch.randint(-1 if n > 1 else 0, classes, (n,), generator=g, device="cuda")
    check_gradients(ops, x, w, labels, torch.rand(n, generator=g, device="cuda"))


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("n", [3, 40, 300, 4100])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=NAME.get)
def test_the_gradient_of_a_row_without_a_label_is_zero_whatever_the_classes_hold(ops, dtype, n, value):
    g = gen(n)
    x, w = normal(g, n, 64, dtype), normal(g, 3100, 64, dtype)
    w[7, 3] = value
    labels = torch.randint(0, 3100, (n,), generator=g, device="cuda", dtype=torch.int32)
    labels[n // 2] = -5
    loss, dx, _ = ops.softmax_loss_grad(x, w, labels, torch.ones(n, device="cuda"))
    assert not dx[n // 2].any() and float(loss[n // 2]) == 0.0
    assert torch.isnan(dx[0]).any()                      # (that of the others is hidden nowhere)
