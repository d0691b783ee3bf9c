"""The training operators against their definitions in 64 bits, at the sizes, types, strides and values where they can go wrong."""
import math

import pytest
import torch

import train_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
NAME = {F32: "f32", BF16: "bf16", F16: "f16"}


@pytest.fixture(scope="module")
def ops():
    import paper_1909_04885_amd as chicle
    return chicle.TrainOps("cuda:0")


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows(g, n, d, dtype, extra=0, shift=0, spread=1.0):
    """n rows of d inside a buffer with longer rows, `shift` values into it."""
    buffer = (torch.randn(n, shift + d + extra, generator=g, device="cuda") * spread).to(dtype)
    return buffer[:, shift:shift + d]


# ---- softmax loss ----------------------------------------------------------------------------------------------------

def check_loss(ops, x, w, labels, weight):
    r = ref.softmax_loss(x, w, labels, weight)
    loss, lse = ops.softmax_loss(x, w, labels)
    has = r["has"]
    ref.within(loss, r["loss"], torch.where(has, r["off_loss"], torch.zeros_like(r["off_loss"])), "loss")
    ref.within(lse[has], r["lse"][has], r["off_lse"][has], "lse")
    loss2, dx, dw = ops.softmax_loss_grad(x, w, labels, weight)
    assert torch.equal(loss, loss2)
    assert dx.dtype == x.dtype and dw.dtype == w.dtype
    ref.within(dx, r["dx"], r["off_dx"], "dx")
    ref.within(dw, r["dw"], r["off_dw"], "dw")
    assert not dx[~has].any()
    ops.sync()
    return dx, dw


@pytest.mark.parametrize("n, d, classes, extra, shift", [
    (1, 64, 1, 0, 0), (1, 1, 2, 0, 0), (1, 200, 1000, 0, 0), (2, 64, 255, 0, 0), (3, 65, 257, 1, 0), (7, 63, 300, 0, 1), (16, 128, 513, 0, 0),
    (17, 100, 700, 3, 5), (64, 64, 640, 0, 0), (65, 192, 1000, 8, 0), (100, 250, 2000, 6, 0), (128, 512, 1024, 0, 0), (129, 320, 777, 0, 3), (257, 96, 4111, 0, 0),
    (600, 130, 3001, 0, 0), (2500, 64, 500, 0, 0),
    (24, 1030, 900, 2, 0), (70, 1100, 300, 0, 0), (96, 600, 500, 0, 0), (97, 700, 515, 0, 1), (130, 1024, 900, 0, 0), (300, 2050, 700, 0, 0), (64, 2048, 40, 0, 0)])
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_softmax_loss(ops, dtype, n, d, classes, extra, shift):
    print("\ncase softmax_loss", NAME[dtype], n, d, classes, extra, shift, flush=True)
    g = gen(n + d + classes)
    x, w = rows(g, n, d, dtype, extra, shift), rows(g, classes, d, dtype, extra, shift, 2.0 / math.sqrt(d))
    labels = torch.randint(0, classes, (n,), generator=g, device="cuda", dtype=torch.int32 if n % 2 else torch.int64)
    if n > 2:
        labels[torch.rand(n, generator=g, device="cuda") < 0.2] = -1
    weight = torch.rand(n, generator=g, device="cuda") * (64.0 / n)
    check_loss(ops, x, w, labels, weight)


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_softmax_loss_over_several_pieces_of_the_classes(ops, dtype):
    """More rows than one piece of the classes has room for beside them."""
    n, d, classes = 40000 if dtype != F32 else 14000, 16, 9000
    print("\ncase softmax_loss pieces", NAME[dtype], n, d, classes, flush=True)
    g = gen(5)
    x, w = rows(g, n, d, dtype), rows(g, classes, d, dtype, 0, 0, 0.5)
    labels = torch.randint(-1, classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    check_loss(ops, x, w, labels, torch.full((n,), 1.0 / n, device="cuda"))


@pytest.mark.parametrize("dtype", [BF16, F16], ids=NAME.get)
def test_softmax_loss_whose_last_classes_are_less_than_a_round_of_tiles(ops, dtype):
    n, d, classes = 1100, 70, 70001
    print("\ncase softmax_loss last tiles", NAME[dtype], n, d, classes, flush=True)
    g = gen(7)
    x, w = rows(g, n, d, dtype), rows(g, classes, d, dtype, 0, 0, 0.3)
    labels = torch.randint(-1, classes, (n,), generator=g, device="cuda")
    labels[:50] = torch.arange(classes - 50, classes, device="cuda")
    check_loss(ops, x, w, labels, torch.rand(n, generator=g, device="cuda"))


def test_softmax_loss_over_several_pieces_of_the_rows(ops):
    """In 32 bits: more classes than the kept logits have room for beside all rows."""
    n, d, classes = 700, 16, 500001
    print("\ncase softmax_loss row pieces", n, d, classes, flush=True)
    g = gen(6)
    x, w = rows(g, n, d, F32), rows(g, classes, d, F32, 0, 0, 0.5)
    labels = torch.randint(-1, classes, (n,), generator=g, device="cuda")
    check_loss(ops, x, w, labels, torch.rand(n, generator=g, device="cuda"))


def test_softmax_loss_of_more_rows_than_a_second_grid_dimension_holds(ops):
    g = gen(31)
    x, w = rows(g, 70001, 5, F32), rows(g, 3, 5, F32)
    check_loss(ops, x, w, torch.randint(0, 3, (70001,), generator=g, device="cuda", dtype=torch.int32), torch.rand(70001, generator=g, device="cuda") / 70001)


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_softmax_loss_no_row_has_a_label(ops, dtype):
    g = gen(3)
    x, w = rows(g, 70, 64, dtype), rows(g, 300, 64, dtype)
    x[3], x[60] = float("nan"), float("inf")
    labels = torch.full((70,), -100, device="cuda", dtype=torch.int64)
    loss, dx, dw = ops.softmax_loss_grad(x, w, labels, torch.full((70,), float("inf"), device="cuda"))
    assert not loss.any() and not dx.any() and not dw.any()
    ops.sync()


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
@pytest.mark.parametrize("n", [5, 40, 300])
def test_rows_without_a_label_count_nowhere_whatever_they_hold(ops, dtype, n):
    g = gen(n)
    x, w = rows(g, n, 96, dtype), rows(g, 500, 96, dtype, 0, 0, 0.1)
    labels = torch.randint(0, 500, (n,), generator=g, device="cuda", dtype=torch.int32)
    weight = torch.rand(n, generator=g, device="cuda")
    for at, value in ((1, float("nan")), (3, float("inf")), (n - 1, -float("inf"))):
        labels[at], x[at], weight[at] = -1 - at, value, value
    check_loss(ops, x, w, labels, weight)


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_classes_masked_by_the_lowest_value(ops, dtype):
    """x carries a one in a column where masked classes hold the type's lowest value: their probability is zero, and nothing is NaN."""
    g = gen(8)
    n, d, classes = 90, 72, 700
    x, w = rows(g, n, d, dtype), rows(g, classes, d, dtype, 0, 0, 0.2)
    x[:, 5] = 1.0
    w[:, 5] = 0.0
    masked = torch.rand(classes, generator=g, device="cuda") < 0.5
    masked[512:] = True                                  # a whole tile of them
    w[masked] = 0.0
    w[masked, 5] = torch.finfo(dtype).min
    labels = torch.where(masked, -1, torch.arange(classes, device="cuda"))
    labels = labels[labels >= 0][:n].to(torch.int32)
    weight = torch.full((n,), 1.0 / n, device="cuda")
    loss, lse = ops.softmax_loss(x, w, labels)
    keep = (~masked).nonzero()[:, 0]
    back = torch.full((classes,), -1, device="cuda", dtype=torch.int64)
    back[keep] = torch.arange(keep.numel(), device="cuda")
    r = ref.softmax_loss(x, w[keep], back[labels.long()].to(torch.int32), weight)
    ref.within(loss, r["loss"], r["off_loss"])
    ref.within(lse, r["lse"], r["off_lse"])
    _, dx, dw = ops.softmax_loss_grad(x, w, labels, weight)
    ref.within(dx, r["dx"], r["off_dx"])
    ref.within(dw[keep], r["dw"], r["off_dw"])
    assert not dw[masked].any()


@pytest.mark.parametrize("dtype", [BF16, F16], ids=NAME.get)
@pytest.mark.parametrize("n", [30, 500])
def test_a_weight_that_all_rows_share_is_not_rounded(ops, dtype, n):
    """One weight that is no power of two: what is left is the rounding of the gradients, and that of probabilities, to no side.  A weight
    rounded with its row's gradient would take all of dw off by the same part, up to the type's unit round-off."""
    g = gen(n)
    x, w = rows(g, n, 64, dtype), rows(g, 4000, 64, dtype, 0, 0, 0.2)
    labels = torch.randint(0, 4000, (n,), generator=g, device="cuda", dtype=torch.int32)
    u = ref.U[dtype]
    weight = torch.full((n,), (1 + 0.45 * u) * 2.0 ** -4, device="cuda")   # (rounds down to 2^-4)
    r = ref.softmax_loss(x, w, labels, weight)
    _, dx, dw = ops.softmax_loss_grad(x, w, labels, weight)
    for got, want in ((dx, r["dx"]), (dw, r["dw"])):
        along = float((got.double() * want).sum() / (want * want).sum())   # thousands of roundings to either side, each below u / 2
        assert abs(along - 1) < 0.15 * u, along


def test_large_logits_neither_overflow_nor_vanish(ops):
    g = gen(9)
    x, w = rows(g, 50, 64, F32, 0, 0, 30.0), rows(g, 333, 64, F32, 0, 0, 30.0)
    labels = torch.randint(0, 333, (50,), generator=g, device="cuda", dtype=torch.int32)
    check_loss(ops, x, w, labels, torch.ones(50, device="cuda"))


def test_infinities_in_rows_with_labels_are_not_hidden(ops):
    g = gen(10)
    x, w = rows(g, 40, 64, BF16), rows(g, 100, 64, BF16)
    x[7, 3] = float("nan")
    labels = torch.zeros(40, device="cuda", dtype=torch.int32)
    loss, dx, dw = ops.softmax_loss_grad(x, w, labels, torch.ones(40, device="cuda"))
    assert torch.isnan(loss[7]) and not torch.isnan(loss[torch.arange(40, device="cuda") != 7]).any()
    assert torch.isnan(dx[7]).all() and torch.isnan(dw).any()


def test_a_label_past_the_end_is_none_and_reported(ops):
    import paper_1909_04885_amd as chicle
    g = gen(11)
    x, w = rows(g, 20, 64, BF16), rows(g, 100, 64, BF16)
    labels = torch.arange(20, device="cuda", dtype=torch.int64)
    labels[4], labels[9] = 100, 1 << 40
    weight = torch.ones(20, device="cuda")
    loss, dx, dw = ops.softmax_loss_grad(x, w, labels, weight)
    with pytest.raises(chicle.ChicleError, match="label"):
        ops.sync()
    ops.sync()                                           # said once
    labels[4] = labels[9] = -1
    other = ops.softmax_loss_grad(x, w, labels, weight)
    assert all(torch.equal(a, b) for a, b in zip((loss, dx, dw), other))


def test_softmax_loss_gradient_against_differences_of_the_loss(ops):
    """Central differences of 32-bit losses in double: h^2 times a third derivative below 1, and the loss's own error over h."""
    g = gen(12)
    n, d, classes, h = 37, 40, 211, 2.0 ** -6
    x, w = rows(g, n, d, F32), rows(g, classes, d, F32, 0, 0, 0.3)
    labels = torch.randint(0, classes, (n,), generator=g, device="cuda", dtype=torch.int32)
    weight = torch.full((n,), 1.0 / n, device="cuda")
    _, dx, dw = ops.softmax_loss_grad(x, w, labels, weight)
    v, u = torch.randn_like(x) / math.sqrt(d), torch.randn_like(w) / math.sqrt(d)

    def total(x, w):
        return float((weight.double() * ops.softmax_loss(x, w, labels)[0].double()).sum())

    bound = h * h + 64 * 2.0 ** -24 / h
    assert abs((total(x + h * v, w) - total(x - h * v, w)) / (2 * h) - float((dx.double() * v.double()).sum())) < bound
    assert abs((total(x, w + h * u) - total(x, w - h * u)) / (2 * h) - float((dw.double() * u.double()).sum())) < bound


def test_softmax_loss_of_no_rows(ops):
    w = torch.randn(50, 24, device="cuda")
    empty, none = torch.empty(0, 24, device="cuda"), torch.empty(0, device="cuda", dtype=torch.int32)
    assert ops.softmax_loss(empty, w, none)[0].shape == (0,)
    loss, dx, dw = ops.softmax_loss_grad(empty, w, none, torch.empty(0, device="cuda"))
    assert loss.shape == (0,) and dx.shape == (0, 24) and dw.shape == (50, 24) and not dw.any()


def test_half_precision_keeps_gradients_of_very_uneven_weights(ops):
    g = gen(13)
    x, w = rows(g, 200, 64, F16), rows(g, 3000, 64, F16, 0, 0, 0.2)
    labels = torch.randint(0, 3000, (200,), generator=g, device="cuda", dtype=torch.int32)
    for scale in (1e-3, 1.0, 4096.0):
        check_loss(ops, x, w, labels, torch.rand(200, generator=g, device="cuda") * scale)


def test_classes_past_32_bit_offsets(ops):
    n, d, classes = 3, 2048, 1100000
    print("\ncase softmax_loss", n, d, classes, flush=True)
    g = gen(14)
    x = rows(g, n, d, BF16)
    w = torch.empty(classes, d, dtype=BF16, device="cuda").normal_(0, 0.02, generator=g)
    labels = torch.tensor([classes - 1, 5, classes // 2], device="cuda", dtype=torch.int32)
    loss, dx, dw = ops.softmax_loss_grad(x, w, labels, torch.ones(n, device="cuda"))
    z = torch.cat([x.float() @ w[i:i + 100000].float().t() for i in range(0, classes, 100000)], 1).double()
    lse = torch.logsumexp(z, 1)
    assert torch.allclose(loss.double(), lse - z[torch.arange(n), labels.long()], atol=1e-4, rtol=0)
    p = torch.exp(z - lse[:, None])
    p[torch.arange(n), labels.long()] -= 1
    for a in (0, classes // 2 - 5, classes - 1000):      # products of three terms: rounded G and rounded sums
        want, mass = p[:, a:a + 1000].t().contiguous() @ x.double(), p[:, a:a + 1000].abs().t().contiguous() @ x.double().abs()
        ref.within(dw[a:a + 1000], want, 4 * ref.U[BF16] * mass + 1e-12, "dw")
    del w, dw


# ---- layer norm ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n, d, extra, shift", [
    (1, 1, 0, 0), (3, 2, 0, 0), (5, 7, 1, 0), (1, 64, 0, 0), (100, 16, 0, 0), (33, 48, 5, 3), (1000, 129, 0, 1), (9, 512, 0, 0), (65, 513, 3, 0), (3, 1024, 8, 0),
    (70, 1537, 3, 0), (4, 2048, 0, 0), (6, 2049, 0, 7), (5, 4096, 0, 0), (3, 8191, 0, 0), (2, 16384, 0, 0), (3, 16385, 0, 1), (2, 40003, 0, 0), (4000, 24, 0, 0)])
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_layer_norm(ops, dtype, n, d, extra, shift):
    print("\ncase layer_norm", NAME[dtype], n, d, extra, shift, flush=True)
    g = gen(n + d)
    x = rows(g, n, d, dtype, extra, shift, 2.0)
    gamma, beta = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dtype), torch.randn(d, generator=g, device="cuda").to(dtype)
    r = ref.layer_norm(x, gamma, beta, 1e-5)
    y, mean, rstd = ops.layer_norm(x, gamma, beta, 1e-5)
    for name, got in (("y", y), ("mean", mean), ("rstd", rstd)):
        ref.within(got, r[name], r["off_" + name], name)
    dy = rows(g, n, d, dtype, shift, extra)
    b = ref.layer_norm_grad(dy, x, gamma, mean, rstd)
    for name, got in zip(("dx", "dgamma", "dbeta"), ops.layer_norm_grad(dy, x, gamma, mean, rstd)):
        assert got.dtype == dtype
        ref.within(got, b[name], b["off_" + name], name)


@pytest.mark.parametrize("n, d", [(5000, 100), (3000, 1000), (20000, 64), (2111, 4097)])
def test_layer_norm_grad_of_many_rows(ops, n, d):
    g = gen(n)
    x, dy, gamma = rows(g, n, d, BF16), rows(g, n, d, BF16), torch.rand(d, generator=g, device="cuda").to(BF16)
    _, mean, rstd = ops.layer_norm(x, gamma, gamma)
    b = ref.layer_norm_grad(dy, x, gamma, mean, rstd)
    first = ops.layer_norm_grad(dy, x, gamma, mean, rstd)
    for name, got in zip(("dx", "dgamma", "dbeta"), first):
        ref.within(got, b[name], b["off_" + name], name)
    assert all(torch.equal(a, c) for a, c in zip(first, ops.layer_norm_grad(dy, x, gamma, mean, rstd)))


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_layer_norm_of_constant_and_far_off_rows(ops, dtype):
    x = torch.randn(12, 300, device="cuda").to(dtype)
    x[3] = 7.0
    x[4] = 0.0
    x[5] = x[5] + 1000.0
    gamma = beta = torch.ones(300, device="cuda", dtype=dtype)
    r = ref.layer_norm(x, gamma, beta, 1e-5)
    y, mean, rstd = ops.layer_norm(x, gamma, beta, 1e-5)
    for name, got in (("y", y), ("mean", mean), ("rstd", rstd)):
        ref.within(got, r[name], r["off_" + name], name)
    assert torch.equal(y[4], beta)


def test_layer_norm_keeps_what_is_no_number_in_its_row(ops):
    x = torch.randn(40, 200, device="cuda")
    clean = ops.layer_norm(x, x[0], x[1])[0]
    x[7, 5], x[20, 0] = float("nan"), float("inf")
    y = ops.layer_norm(x, clean[0] * 0 + 1, x[1])[0]
    bad = torch.isnan(y).any(1)
    assert bad[7] and bad[20] and int(bad.sum()) == 2


def test_layer_norm_gradient_against_differences(ops):
    g = gen(4)
    n, d, h = 21, 130, 2.0 ** -6
    x, dy = rows(g, n, d, F32), rows(g, n, d, F32)
    gamma, beta = torch.rand(d, generator=g, device="cuda") + 0.5, torch.rand(d, generator=g, device="cuda")
    _, mean, rstd = ops.layer_norm(x, gamma, beta)
    dx, dgamma, dbeta = ops.layer_norm_grad(dy, x, gamma, mean, rstd)

    def total(x, gamma, beta):
        return float((dy.double() * ops.layer_norm(x, gamma, beta)[0].double()).sum())

    v, q = torch.randn_like(x), torch.randn_like(gamma)
    # third derivatives of a row's normalised values are of order one in units of its own spread; sums of n d terms of order one
    bound = 8 * h * h * math.sqrt(n * d) + 64 * 2.0 ** -24 * math.sqrt(n * d) / h
    assert abs((total(x + h * v, gamma, beta) - total(x - h * v, gamma, beta)) / (2 * h) - float((dx.double() * v).sum())) < bound
    assert abs((total(x, gamma + h * q, beta) - total(x, gamma - h * q, beta)) / (2 * h) - float((dgamma.double() * q).sum())) < bound
    assert abs((total(x, gamma, beta + h * q) - total(x, gamma, beta - h * q)) / (2 * h) - float((dbeta.double() * q).sum())) < bound


def test_layer_norm_of_no_rows(ops):
    e, v = torch.empty(0, 30, device="cuda"), torch.ones(30, device="cuda")
    y, mean, rstd = ops.layer_norm(e, v, v)
    assert y.shape == (0, 30)
    dx, dgamma, dbeta = ops.layer_norm_grad(e, e, v, mean, rstd)
    assert dx.shape == (0, 30) and not dgamma.any() and not dbeta.any()


# ---- table lookup ----------------------------------------------------------------------------------------------------

def token_ids(g, n, n_rows, kind, wide):
    if kind == "one":
        ids = torch.full((n,), n_rows // 2, device="cuda", dtype=torch.int64)
    elif kind == "zipf":
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        ids = ((n_rows + 1) ** u).long().sub_(1).clamp_(0, n_rows - 1)
    elif kind == "down":
        ids = torch.arange(n, device="cuda").flip(0) % n_rows
    else:
        ids = torch.randint(0, n_rows, (n,), generator=g, device="cuda")
        ids[torch.rand(n, generator=g, device="cuda") < 0.3] = -1
    return ids.to(torch.int64 if wide else torch.int32)


@pytest.mark.parametrize("n, d, n_rows", [(1, 1, 1), (1, 64, 9), (5, 7, 3), (100, 48, 1000), (333, 1001, 77), (20, 5000, 50), (5001, 16, 70000)])
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_embed(ops, dtype, n, d, n_rows):
    g = gen(n + d)
    ids = token_ids(g, n, n_rows, "some", n % 2 == 0)
    for extra, shift in ((0, 0), (3, 1)):
        table = rows(g, n_rows, d, dtype, extra, shift)
        got = ops.embed(table, ids, 0.37)
        want = torch.where(ids[:, None] >= 0, table.double()[ids.long().clamp(min=0)] * 0.37, torch.zeros((), dtype=torch.float64, device="cuda"))
        ref.within(got, want, (ref.U[dtype] + 2 * ref.U32) * want.abs() + ref.TINY[dtype])
    assert torch.equal(ops.embed(table, ids.reshape(1, -1, 1))[0, :, 0], torch.where(ids[:, None] >= 0, table[ids.long().clamp(min=0)], torch.zeros_like(table[:1])))


@pytest.mark.parametrize("n, d, n_rows", [
    (1, 1, 1), (1, 64, 1000), (31, 3, 5), (32, 40, 4), (33, 250, 100), (64, 16, 1), (1000, 300, 200), (4096, 24, 3000), (4097, 24, 3000), (6144, 100, 1023),
    (10000, 17, 1024), (20011, 129, 50021), (70000, 16, 1000000), (3000, 2100, 500)])
@pytest.mark.parametrize("kind", ["some", "zipf", "one", "down"])
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_embed_grad(ops, dtype, kind, n, d, n_rows):
    print("\ncase embed_grad", NAME[dtype], kind, n, d, n_rows, flush=True)
    g = gen(n + d + n_rows)
    ids = token_ids(g, n, n_rows, kind, n % 2 == 0)
    dout = rows(g, n, d, dtype, n % 3, d % 4)
    want, off = ref.embed_grad(ids, dout, n_rows, 1.7)
    got = ops.embed_grad(ids, dout, n_rows, 1.7)
    ref.within(got, want, off)
    assert torch.equal(got, ops.embed_grad(ids, dout, n_rows, 1.7))     # one order of the sums, whatever the timing
    into = rows(g, n_rows, d, dtype, 3, 1)
    before = into.clone()
    want, off = ref.embed_grad(ids, dout, n_rows, 1.7, into)
    assert ops.embed_grad(ids, dout, n_rows, 1.7, into) is into
    ref.within(into, want, off)
    untouched = torch.ones(n_rows, dtype=torch.bool, device="cuda")
    untouched[ids[ids >= 0].long()] = False
    assert torch.equal(into[untouched], before[untouched])
    ops.sync()


def test_embed_grad_of_many_wide_rows(ops):
    g = gen(32)
    n, d, n_rows = 2 ** 17 + 45, 1034, 3001
    ids = token_ids(g, n, n_rows, "zipf", False)
    dout = rows(g, n, d, BF16)
    want, off = ref.embed_grad(ids, dout, n_rows, 0.6)
    ref.within(ops.embed_grad(ids, dout, n_rows, 0.6), want, off)


def test_embed_without_tokens(ops):
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert ops.embed(torch.ones(3, 5, device="cuda"), none).shape == (0, 5)
    dout = torch.empty(0, 5, device="cuda")
    assert not ops.embed_grad(none, dout, 7).any() and ops.embed_grad(none, dout, 7).shape == (7, 5)
    into = torch.ones(7, 5, device="cuda")
    assert torch.equal(ops.embed_grad(none, dout, 7, into=into), torch.ones(7, 5, device="cuda"))
    none = torch.full((50,), -3, dtype=torch.int64, device="cuda")
    assert not ops.embed_grad(none, torch.full((50, 5), float("nan"), device="cuda"), 7).any()


def test_tokens_past_the_table_are_none_and_reported(ops):
    import paper_1909_04885_amd as chicle
    table = torch.randn(10, 24, device="cuda")
    for n in (6, 9000):
        ids = torch.arange(n, device="cuda", dtype=torch.int64) % 10
        ids[2], ids[4] = 10, 1 << 35
        out = ops.embed(table, ids)
        with pytest.raises(chicle.ChicleError, match="token"):
            ops.sync()
        dout = torch.randn(n, 24, device="cuda")
        got = ops.embed_grad(ids, dout, 10)
        with pytest.raises(chicle.ChicleError, match="token"):
            ops.sync()
        ids[2] = ids[4] = -1
        assert torch.equal(out, ops.embed(table, ids)) and not out[2].any()
        assert torch.equal(got, ops.embed_grad(ids, dout, 10))
        ops.sync()


def test_rows_past_32_bit_offsets(ops):
    n_rows, d = 1100000, 2048
    table = torch.empty(n_rows, d, dtype=BF16, device="cuda")
    ids = torch.tensor([n_rows - 1, 3, n_rows - 1, 0, n_rows // 2 + 77], device="cuda")
    table[ids] = torch.randn(5, d, device="cuda").to(BF16)
    assert torch.equal(ops.embed(table, ids), table[ids])
    del table
    dout = torch.randn(5, d, device="cuda").to(BF16)
    got = ops.embed_grad(ids, dout, n_rows)
    assert int((got != 0).any(1).sum()) == 4
    assert torch.equal(got[n_rows // 2 + 77], dout[4])
    want = dout[0].float() + dout[2].float()
    assert torch.equal(got[n_rows - 1], want.to(BF16))
    x = got                                              # rows of layer norm, as many
    x[-2:] = torch.randn(2, d, device="cuda").to(BF16)
    one = torch.ones(d, device="cuda", dtype=BF16)
    y = ops.layer_norm(x, one, one)[0]
    assert torch.equal(y[-2:], ops.layer_norm(x[-2:], one, one)[0])


# ---- clipping --------------------------------------------------------------------------------------------------------

def norm_of(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


@pytest.mark.parametrize("shapes", [[(1,)], [(0,), (3, 0), (5,)], [(1000,)], [(7, 11), (1,), (333,), (64, 64)], [(100003,), (2,)], [(5,)] * 250, [(3000000,)],
                                    [(i,) for i in range(400)]], ids=lambda s: "%dx%s" % (len(s), s[0]))
@pytest.mark.parametrize("dtype", [F32, BF16, F16, None], ids=lambda t: NAME.get(t, "mixed"))
def test_clip_grads(ops, dtype, shapes):
    g = gen(len(shapes))
    grads = [(torch.randn(s, generator=g, device="cuda") * 3).to(dtype or TYPES[k % 3]) for k, s in enumerate(shapes)]
    norm = norm_of(grads)
    for max_norm in (0.31 * norm, 3 * norm + 1, 0.0):
        factor = min(1.0, max_norm / (norm + 1e-6))
        out = [torch.full_like(t, 5.0) for t in grads]
        kept = [t.clone() for t in grads]
        got = ops.clip_grads(grads, max_norm, out)
        assert all(torch.equal(a, b) for a, b in zip(grads, kept))
        # squares and their sums are in double: what is left is the rounding of the norm and of the factor
        assert abs(float(got) - norm) <= 2 * ref.U32 * norm
        for t, o in zip(grads, out):
            want = t.double() * factor
            ref.within(o, want, (ref.U[t.dtype] + 8 * ref.U32) * want.abs() + ref.TINY[t.dtype])
        assert torch.equal(ops.clip_grads(grads, max_norm), got)
        assert all(torch.equal(a, b) for a, b in zip(grads, out))
        grads = kept
    assert torch.equal(ops.grad_norm(grads), ops.clip_grads(grads, 0.0))


def test_clip_grads_of_nothing(ops):
    assert float(ops.clip_grads([], 1.0)) == 0.0 and float(ops.grad_norm([])) == 0.0
    z = torch.zeros(100, device="cuda")
    assert float(ops.clip_grads([z], 1.0)) == 0.0 and not z.any()


def test_clip_grads_at_any_offset(ops):
    base = torch.randn(5000, device="cuda").to(BF16)
    for a, b in ((1, 2), (3, 4000), (7, 5000)):
        part = base[a:b]
        got = ops.clip_grads([part], 1e9, [torch.empty_like(part)])
        assert abs(float(got) - norm_of([part])) <= 2 * ref.U32 * norm_of([part])


def test_squares_that_32_bits_do_not_hold(ops):
    t = torch.full((1000,), 1e30, device="cuda")
    got = float(ops.clip_grads([t], 1.0))
    assert abs(got / (1e30 * math.sqrt(1000)) - 1) < 1e-6
    assert torch.allclose(t, torch.full_like(t, 1 / math.sqrt(1000)), rtol=1e-6)
    t = torch.full((1000,), 1e-30, device="cuda")
    assert abs(float(ops.grad_norm([t])) / (1e-30 * math.sqrt(1000)) - 1) < 1e-6


def test_a_norm_that_is_no_number(ops):
    a, b = torch.ones(300, device="cuda"), torch.ones(10, device="cuda")
    a[5] = float("inf")
    assert float(ops.clip_grads([a, b], 1.0)) == float("inf")
    assert torch.isnan(a[5]) and not a[:5].any() and not b.any()
    b[3] = float("nan")
    assert math.isnan(float(ops.clip_grads([b], 1.0))) and torch.isnan(b).all()


# ---- how they are called ---------------------------------------------------------------------------------------------

def test_refusals_of_the_binding(ops):
    import paper_1909_04885_amd as chicle
    x, w = torch.randn(4, 8, device="cuda"), torch.randn(10, 8, device="cuda")
    labels, weight, v = torch.zeros(4, device="cuda", dtype=torch.int32), torch.ones(4, device="cuda"), torch.ones(8, device="cuda")
    bad = [
        lambda: ops.softmax_loss(x.cpu(), w, labels), lambda: ops.softmax_loss(x.double(), w, labels), lambda: ops.softmax_loss(x, w.to(BF16), labels),
        lambda: ops.softmax_loss(x, w[:, :7], labels), lambda: ops.softmax_loss(x, w, labels[:3]), lambda: ops.softmax_loss(x, w, labels.float()),
        lambda: ops.softmax_loss(x.t(), w, labels), lambda: ops.softmax_loss(x[0], w, labels), lambda: ops.softmax_loss(x, w[:0], labels),
        lambda: ops.softmax_loss(x[:1].expand(4, 8), w, labels), lambda: ops.softmax_loss_grad(x, w, labels, weight.double()),
        lambda: ops.softmax_loss_grad(x, w, labels, weight[:2]), lambda: ops.embed(w, labels.float()), lambda: ops.embed(w.t(), labels),
        lambda: ops.embed_grad(labels, x[:3], 10), lambda: ops.embed_grad(labels, x, 0), lambda: ops.embed_grad(labels, x, 10, into=w[:9]),
        lambda: ops.embed_grad(labels, x, 10, into=w.to(F16)), lambda: ops.layer_norm(x, v[:7], v), lambda: ops.layer_norm(x, v, v.to(BF16)),
        lambda: ops.layer_norm(x, v, v, -1.0), lambda: ops.layer_norm_grad(x[:3], x, v, weight, weight), lambda: ops.layer_norm_grad(x, x, v, weight, weight[:2]),
        lambda: ops.clip_grads([x.t()], 1.0), lambda: ops.clip_grads([x], 1.0, []), lambda: ops.clip_grads([x], 1.0, [w]), lambda: ops.clip_grads([x], -1.0),
        lambda: ops.clip_grads([x.long()], 1.0)]
    for k, call in enumerate(bad):
        with pytest.raises(chicle.ChicleError):
            call()
            pytest.fail("call %d was not refused" % k)


def one_step(ops, ids, table, gamma, beta, w, labels, weight):
    x = ops.embed(table, ids, 2.0)
    y, mean, rstd = ops.layer_norm(x, gamma, beta)
    loss, dy, dw = ops.softmax_loss_grad(y, w, labels, weight)
    dx, dgamma, dbeta = ops.layer_norm_grad(dy, x, gamma, mean, rstd)
    dtable = ops.embed_grad(ids, dx, table.shape[0], 2.0)
    grads = [dtable, dgamma, dbeta, dw]
    out = [torch.empty_like(t) for t in grads]
    norm = ops.clip_grads(grads, 0.5, out)
    return [loss, norm] + out


def step_inputs(dtype, seed, n=600, d=100, n_rows=5000, classes=900):
    g = gen(seed)
    return [torch.randint(0, n_rows, (n,), generator=g, device="cuda"), rows(g, n_rows, d, dtype), rows(g, 1, d, dtype)[0].contiguous(),
            rows(g, 1, d, dtype)[0].contiguous(), rows(g, classes, d, dtype, 0, 0, 0.2), torch.randint(-1, classes, (n,), generator=g, device="cuda"),
            torch.full((n,), 1 / n, device="cuda")]


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_on_a_stream_of_the_callers(ops, dtype):
    args = step_inputs(dtype, 2)
    want = one_step(ops, *args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        outs = [one_step(ops, *args) for _ in range(3)]
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("dtype", [F32, F16], ids=NAME.get)
def test_captured_into_a_graph(ops, dtype):
    """Replayed several times on new inputs, with other work in between, and compared with the same calls outside the graph."""
    args = step_inputs(dtype, 3, n=5000)
    one_step(ops, *args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = one_step(ops, *args)
    for seed in (4, 5, 6):
        for a, b in zip(args, step_inputs(dtype, seed, n=5000)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = one_step(ops, *args)
        torch.randn(1000, 1000, device="cuda").sum().item()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed
