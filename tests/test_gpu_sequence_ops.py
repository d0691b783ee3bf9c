"""The operators of layers over sequences against their definitions in 64 bits, at the sizes, types, strides and values where they can go wrong."""
import pytest
import torch

import sequence_reference as ref
from train_reference import TINY, U, U32, within

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
NAME = {F32: "f32", BF16: "bf16", F16: "f16"}
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ops():
    import paper_1909_04885_amd as chicle
    return chicle.TrainOps("cuda:0")


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows(g, n, d, dtype, extra=0, shift=0, spread=1.0, mean=0.0):
    """n rows of d inside a buffer with longer rows, `shift` values into it."""
    buffer = (torch.randn(n, shift + d + extra, generator=g, device="cuda") * spread + mean).to(dtype)
    return buffer[:, shift:shift + d]


# ---- rows in 8 bits ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n, d, extra, shift", [(0, 40, 0, 0), (1, 1, 0, 0), (1, 4096, 0, 0), (3, 7, 2, 1), (5, 31, 0, 0), (4, 32, 0, 0), (70, 33, 3, 5), (333, 250, 6, 0),
                                                (1000, 1537, 0, 1), (77, 5000, 0, 0), (4100, 64, 0, 0)])
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_pack8(ops, dtype, n, d, extra, shift):
    print("\ncase pack8", NAME[dtype], n, d, extra, shift, flush=True)
    g = gen(n + d)
    x = rows(g, n, d, dtype, extra, shift) * torch.exp(2 * torch.randn(n, 1, generator=g, device="cuda")).to(dtype)
    p = ops.pack8(x)
    q, byte = ref.pack(x)
    assert torch.equal(p.values.double(), q) and torch.equal(p.scales, byte)
    for out in TYPES:
        v = ops.unpack8(p, out)
        assert v.dtype == out and torch.equal(v, ref.unpack(q, byte, d).to(out))
    within(ops.unpack8(p, dtype), x, ref.step_of(byte, d) / 2)


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_pack8_at_the_ends_of_the_range(ops, dtype):
    most, least = torch.finfo(dtype).max, TINY[dtype]
    x = torch.zeros(6, 96, dtype=F32, device="cuda")
    x[0, 3], x[0, 40], x[1, 64:] = most, -most, most
    x[2, :32] = 127.0                                    # on a power's border
    x[2, 32:64], x[2, 40] = 127.0, 127.5
    x[3, :] = least
    x[4, ::2] = -2.0 ** -14
    x = x.to(dtype)
    p = ops.pack8(x)
    q, byte = ref.pack(x)
    q = torch.where((q.abs() == 64) & (x.abs() > most / 2).view(q.shape), q.sign() * 63, q)    # (64 steps would be a power of two past the largest number)
    assert torch.equal(p.values.double(), q) and torch.equal(p.scales, byte)
    v = ops.unpack8(p, dtype)
    assert bool(v.isfinite().all()) and not v[5].any()
    # the largest number is 2^k (1 - U) with 2^k = 64 steps, of which 63 are kept: off by 1 - 64 U steps (the others by half a step)
    within(v, x, ref.step_of(byte, 96) * max(0.5, 1 - 64 * U[dtype]))


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_pack8_groups_that_are_not_finite(ops, dtype):
    x = rows(gen(1), 5, 100, dtype)
    x[0, 5], x[1, 40], x[2, 99], x[3, 64:] = NAN, INF, -INF, NAN
    v = ops.unpack8(ops.pack8(x), dtype)
    bad = torch.zeros(5, 100, dtype=torch.bool, device="cuda")
    bad[0, :32] = bad[1, 32:64] = bad[2, 96:] = bad[3, 64:] = True
    assert torch.equal(v.isnan(), bad)
    within(v[~bad], x[~bad], 4.0 / 127)                  # (half a step of values up to 8)


# ---- root-mean-square norm ---------------------------------------------------------------------------------------------

NORM_SIZES = [(1, 1, 0, 0), (1, 4096, 0, 0), (3, 5, 2, 1), (7, 31, 0, 0), (5, 64, 0, 0), (300, 100, 3, 0), (130, 250, 6, 1), (65, 1000, 0, 0), (33, 1537, 3, 0), (9, 4096, 8, 0),
              (4, 5000, 0, 3), (3, 16384, 0, 0), (5, 20001, 0, 0), (3, 40000, 1, 0), (2100, 40, 0, 0)]


def check_packed(ops, p, want, off, what):
    """A packed result whose 32-bit values are off by `off`: half a step more, and a step of twice the size where those lie at its border."""
    d = want.shape[1]
    _, byte = ref.pack(want.abs() + off)
    within(ops.unpack8(p, F32), want, off + ref.step_of(byte, d) / 2 + 2 * U32 * want.abs(), what)
    assert not p.values[:, d:].any()


@pytest.mark.parametrize("n, d, extra, shift", NORM_SIZES)
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_rms_norm(ops, dtype, n, d, extra, shift):
    print("\ncase rms_norm", NAME[dtype], n, d, extra, shift, flush=True)
    g = gen(n * 7 + d)
    x, res = rows(g, n, d, dtype, extra, shift), rows(g, n, d, dtype, extra, shift, 3.0)
    gamma = rows(g, 1, d, dtype, 0, 0, 0.2, 1.0)[0]
    for residual in (None, res):
        w = ref.rms_norm(x, gamma, residual, 1e-5)
        y, r, rstd, kept = ops.rms_norm(x, gamma, residual)
        assert kept is None and torch.equal(r, w["r"]) and (residual is not None or r is x)
        within(rstd, w["rstd"], w["off_rstd"], "rstd")
        within(y, w["y"], w["off_y"], "y")
        y8, r2, rstd2, kept = ops.rms_norm(x, gamma, residual, y8=True, keep8=True)
        assert torch.equal(r, r2) and torch.equal(rstd, rstd2)
        check_packed(ops, y8, w["y"], w["off_y32"], "y8")
        want = ops.pack8(r.contiguous())
        assert torch.equal(kept.values, want.values) and torch.equal(kept.scales, want.scales)
        y3, _, _, kept2 = ops.rms_norm(x, gamma, residual, keep8=True)
        assert torch.equal(y3, y) and torch.equal(kept2.values, kept.values)
    ops.sync()


@pytest.mark.parametrize("n, d, extra, shift", NORM_SIZES + [(9001, 96, 0, 0), (3000, 1024, 0, 0), (0, 64, 0, 0)])
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_rms_norm_grad(ops, dtype, n, d, extra, shift):
    print("\ncase rms_norm_grad", NAME[dtype], n, d, extra, shift, flush=True)
    g = gen(n * 5 + d)
    r, dy, dr = (rows(g, n, d, dtype, extra, shift, s) for s in (2.0, 1.0, 0.5))
    gamma = rows(g, 1, d, dtype, 0, 0, 0.2, 1.0)[0]
    rstd = ((r.double() ** 2).mean(1) + 1e-5).rsqrt().float()
    p = ops.pack8(r)
    for more in (None, dr):
        for given, values in ((r, r), (p, ref.unpack(p.values, p.scales, d))):
            w = ref.rms_norm_grad(dy, values, gamma, rstd, more)
            dx, dgamma = ops.rms_norm_grad(dy, given, gamma, rstd, more)
            assert dx.dtype == dtype and dgamma.dtype == dtype
            within(dx, w["dx"], w["off_dx"], "dx")
            within(dgamma, w["dgamma"], w["off_dgamma"], "dgamma")


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_rms_norm_keeps_what_is_not_finite_in_its_row(ops, dtype):
    g = gen(2)
    x, gamma = rows(g, 9, 200, dtype), rows(g, 1, 200, dtype)[0]
    clean, _, clean_rstd, _ = ops.rms_norm(x, gamma)
    x[2, 5], x[7, 190] = NAN, INF
    y, _, rstd, _ = ops.rms_norm(x, gamma)
    others = torch.tensor([0, 1, 3, 4, 5, 6, 8], device="cuda")
    assert torch.equal(y[others], clean[others]) and torch.equal(rstd[others], clean_rstd[others])
    assert bool(y[2].isnan().all()) and float(rstd[7]) == 0.0 and bool(y[7, 190].isnan()) and not y[7, :190].any()


# ---- gated recurrence --------------------------------------------------------------------------------------------------

def lengths_of(kind, n):
    if kind == "one":
        return [n]
    if kind == "ones":
        return [1] * n
    out, left, k = [], n, 0
    while left > 0:                                      # short and long ones, every fifth empty
        size = 0 if k % 5 == 2 else min(left, (1, 2, 31, 32, 33, 5, 64, 100, 257)[k % 9])
        out.append(size)
        left -= size
        k += 1
    return out + [0]


def offsets_of(lengths, wide, first=0):
    at = [first]
    for x in lengths:
        at.append(at[-1] + x)
    return at, torch.tensor(at, dtype=torch.int64 if wide else torch.int32, device="cuda")


def scan_case(g, n, d, dtype, extra, shift, lengths, packed, with_h0, ops, first=0):
    f, u = rows(g, n, d, dtype, extra, shift, 2.0, 1.5), rows(g, n, d, dtype, extra, shift)
    at, offsets = offsets_of(lengths, n % 2 == 1, first)
    k = len(lengths)
    h0 = torch.randn(k, d, generator=g, device="cuda") if with_h0 else None
    values = u
    if packed:
        u = ops.pack8(u)
        values = ref.unpack(u.values, u.scales, d)
    return f, u, values, at, offsets, h0


def check_scan(ops, f, u, values, at, offsets, h0, given=True):
    dtype, n = f.dtype, f.shape[0]
    w = ref.scan(f.cpu(), values.cpu(), at, None if h0 is None else h0.cpu())
    y, last, states = ops.gated_scan(f, u, offsets if given else None, h0, last=True, states=True)
    within(y.cpu(), w["h"], w["off"] + U[dtype] * w["h"].abs() + TINY[dtype], "y")
    within(last.cpu(), w["last"], w["off_last"], "last")
    within(states.cpu(), w["before"][::ref.KEPT], w["off_before"][::ref.KEPT], "states")
    y2, no_last, no_states = ops.gated_scan(f, u, offsets if given else None, h0)
    assert torch.equal(y, y2) and no_last is None and no_states is None
    assert not y[at[-1]:].any() and not y[:at[0]].any()
    ops.sync()
    return y, last, states


def check_scan_grad(ops, g, f, u, values, at, offsets, h0, with_dlast, given=True):
    n, d = f.shape
    _, _, states = ops.gated_scan(f, u, offsets if given else None, h0, states=True)
    dy = rows(g, n, d, f.dtype, 3, 1)
    dlast = torch.randn(len(at) - 1, d, generator=g, device="cuda") if with_dlast else None
    w = ref.scan_grad(f.cpu(), values.cpu(), at, None if h0 is None else h0.cpu(), dy.cpu(), None if dlast is None else dlast.cpu())
    df, du, dh0 = ops.gated_scan_grad(f, u, states, dy, offsets if given else None, h0, dlast)
    within(df.cpu(), w["df"], w["off_df"], "df")
    within(du.cpu(), w["du"], w["off_du"], "du")
    assert (dh0 is None) == (h0 is None)
    if h0 is not None:
        within(dh0.cpu(), w["dh0"], w["off_dh0"], "dh0")
    ops.sync()


SCANS = [(1, 1, 0, 0, "one"), (1, 64, 0, 0, "one"), (2, 3, 1, 1, "ones"), (31, 130, 0, 0, "one"), (32, 128, 0, 0, "some"), (33, 129, 2, 1, "some"), (64, 257, 0, 0, "ones"),
         (300, 250, 6, 0, "some"), (129, 1000, 0, 0, "one"), (700, 31, 0, 3, "some"), (257, 2, 0, 0, "one"), (2500, 17, 0, 0, "one"), (5000, 9, 0, 0, "some")]


@pytest.mark.parametrize("with_h0", [False, True])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("n, d, extra, shift, kind", SCANS)
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_gated_scan(ops, dtype, n, d, extra, shift, kind, packed, with_h0):
    print("\ncase gated_scan", NAME[dtype], n, d, extra, shift, kind, packed, with_h0, flush=True)
    g = gen(n + d)
    case = scan_case(g, n, d, dtype, extra, shift, lengths_of(kind, n), packed, with_h0, ops)
    check_scan(ops, *case)
    check_scan_grad(ops, g, *case, with_dlast=with_h0)


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_gated_scan_without_offsets_is_one_sequence(ops, dtype):
    g = gen(4)
    case = scan_case(g, 400, 70, dtype, 0, 0, [400], False, True, ops)
    check_scan(ops, *case, given=False)
    check_scan_grad(ops, g, *case, with_dlast=True, given=False)


@pytest.mark.parametrize("n, first, lengths", [(500, 0, [100, 0, 33]), (500, 40, [100, 0, 33]), (500, 500, [0, 0]), (70, 3, [0]), (300, 0, [0, 0, 0]), (260, 129, [0, 64, 0, 1])])
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_rows_of_no_sequence_get_zeros_whatever_they_hold(ops, dtype, n, first, lengths):
    print("\ncase rows of no sequence", NAME[dtype], n, first, lengths, flush=True)
    g = gen(n + first)
    f, u, values, at, offsets, h0 = scan_case(g, n, 90, dtype, 0, 0, lengths, False, True, ops, first)
    out = torch.ones(n, dtype=torch.bool, device="cuda")
    out[at[0]:at[-1]] = False
    f[out], u[out] = NAN, INF
    y, last, states = ops.gated_scan(f, u, offsets, h0, last=True, states=True)
    dy, dlast = rows(g, n, 90, dtype), torch.randn(len(lengths), 90, generator=g, device="cuda")
    dy[out] = NAN
    df, du, dh0 = ops.gated_scan_grad(f, u, states, dy, offsets, h0, dlast)
    assert not y[out].any() and not df[out].any() and not du[out].any()
    f[out], u[out], dy[out] = 0.0, 0.0, 0.0
    check_scan(ops, f, u, u, at, offsets, h0)
    assert torch.equal(ops.gated_scan(f, u, offsets, h0)[0], y)
    again = ops.gated_scan_grad(f, u, states, dy, offsets, h0, dlast)
    assert all(torch.equal(p, q) for p, q in zip(again, (df, du, dh0)))
    empty = torch.tensor([x == 0 for x in lengths], device="cuda")
    assert torch.equal(last[empty], h0[empty]) and torch.equal(dh0[empty], dlast[empty])


@pytest.mark.parametrize("k", [0, 1, 70])
def test_gated_scan_of_no_rows(ops, k):
    h0, offsets = torch.randn(k, 50, device="cuda"), torch.zeros(k + 1, dtype=torch.int32, device="cuda")
    f = torch.empty(0, 50, device="cuda")
    y, last, states = ops.gated_scan(f, f, offsets, h0, last=True, states=True)
    assert y.shape == (0, 50) and states.shape == (0, 50) and torch.equal(last, h0)
    _, _, dh0 = ops.gated_scan_grad(f, f, states, f, offsets, h0, 2 * h0)
    assert torch.equal(dh0, 2 * h0)
    ops.sync()


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_closed_gates_let_nothing_through_whatever_is_there(ops, dtype):
    """f = +infinity, or the type's largest number, masks a row; f = -infinity forgets what was before."""
    g = gen(6)
    n, d = 400, 70
    f, u = rows(g, n, d, dtype, 0, 0, 1.0, 1.0), rows(g, n, d, dtype)
    big = torch.finfo(dtype).max
    masked = torch.rand(n, d, generator=g, device="cuda") < 0.3
    masked[100:170] = True                               # whole tiles
    f[masked] = torch.where(torch.rand(n, d, generator=g, device="cuda") < 0.5, INF, big).to(dtype)[masked]
    dirty = u.clone()
    dirty[masked] = torch.where(torch.rand(n, d, generator=g, device="cuda") < 0.5, NAN, INF).to(dtype)[masked]
    y, last, states = ops.gated_scan(f, dirty, last=True, states=True)
    clean, clean_last, clean_states = check_scan(ops, f, u, u, [0, n], None, None, given=False)
    assert torch.equal(y, clean) and torch.equal(last, clean_last) and torch.equal(states, clean_states)
    # 32 rows at a time are gone through one after the other, and a closed gate's share is exactly none; what they begin with has come through a product of
    # shares and is a rounding off, to the bounds above
    for lo, hi in ((100, 128), (128, 160), (160, 170)):
        assert torch.equal(y[lo:hi], y[lo].expand(hi - lo, d))
    dy = rows(g, n, d, dtype)
    got, want = ops.gated_scan_grad(f, dirty, states, dy), ops.gated_scan_grad(f, u, states, dy)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and not got[0][masked].any() and not got[1][masked].any()
    # what was before a row that forgets counts nowhere behind it, nor does what comes behind it before
    f, u = rows(g, n, d, dtype, 0, 0, 1.0, 1.0), rows(g, n, d, dtype)
    for at, value in ((37, -INF), (64, -big), (200, -INF)):
        f[at] = value
    clean, _, _ = check_scan(ops, f, u, u, [0, n], None, None, given=False)
    dirty = u.clone()
    dirty[:199, ::2] = NAN
    dirty[5, 1::2] = INF
    y, _, states = ops.gated_scan(f, dirty, states=True)
    assert torch.equal(y[200:], clean[200:]) and bool(y[190:199, ::2].isnan().all())
    assert torch.equal(y[37:, 1::2], clean[37:, 1::2]) and not bool(y[5:37, 1::2].isfinite().any())
    dy = rows(g, n, d, dtype)
    dy[200:, ::3] = NAN
    _, du, _ = ops.gated_scan_grad(f, u, ops.gated_scan(f, u, states=True)[2], dy)
    assert bool(du[200:, ::3].isnan().all()) and bool(du[:200].isfinite().all())


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_values_at_the_ends_of_the_range_do_not_overflow(ops, dtype):
    """States stay between the values that come in, also where these are the type's largest and lowest."""
    g = gen(9)
    big = torch.finfo(dtype).max
    f = rows(g, 200, 40, dtype)
    u = torch.where(torch.rand(200, 40, generator=g, device="cuda") < 0.5, big, -big).to(dtype)
    check_scan(ops, f, u, u, [0, 200], None, None, given=False)


@pytest.mark.parametrize("at", [[0, 50, 40, 100], [-5, 10, 20, 100], [0, 10, 20, 101], [0, 10, 20, 2 ** 31 - 1], [0, -1, 100, 100]])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAME.get)
def test_offsets_that_are_no_rows_are_reported(ops, dtype, at):
    import paper_1909_04885_amd as chicle
    print("\ncase offsets", NAME[dtype], at, flush=True)
    g = gen(1)
    guard = torch.full((300, 40), 7.0, dtype=dtype, device="cuda")
    f, u = rows(g, 100, 40, dtype), rows(g, 100, 40, dtype)
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    h0 = torch.zeros(3, 40, device="cuda")
    _, _, states = ops.gated_scan(f, u, offsets, h0, last=True, states=True)
    with pytest.raises(chicle.ChicleError, match="offset"):
        ops.sync()
    ops.gated_scan_grad(f, u, states, f, offsets, h0, h0)
    with pytest.raises(chicle.ChicleError, match="offset"):
        ops.sync()
    ops.sync()
    assert bool((guard == 7.0).all())


@pytest.mark.parametrize("n, d, extra, shift", [(1, 1, 0, 0), (3, 5, 2, 1), (4, 1024, 0, 0), (70, 250, 6, 3), (9, 5001, 0, 0), (2000, 33, 1, 0), (0, 8, 0, 0)])
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_gated_step_is_the_scan_of_one_row(ops, dtype, n, d, extra, shift):
    g = gen(n + d)
    f, u = rows(g, n, d, dtype, extra, shift, 2.0, 1.0), rows(g, n, d, dtype, extra, shift)
    wide = torch.full((n, d + 7), 3.0, device="cuda")
    state = wide[:, 2:2 + d]
    state.copy_(torch.randn(n, d, generator=g, device="cuda"))
    before = state.clone()
    version = state._version
    y = ops.gated_step(f, u, state)
    want, last, _ = ops.gated_scan(f, u, torch.arange(n + 1, device="cuda"), before, last=True)
    assert torch.equal(y, want) and torch.equal(state, last) and state._version > version
    assert bool((wide[:, :2] == 3.0).all()) and bool((wide[:, 2 + d:] == 3.0).all())
    a, c, s = ref.gates(f)
    exact = a * before.double() + c * u.double()
    within(state, exact, 2 * (ref.gate_off(f) * s * (before.double().abs() + u.double().abs()) + 2 * U32 * (a * before.double().abs() + c * u.double().abs())))


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_a_prompt_in_pieces_and_rows_one_by_one(ops, dtype):
    """What a program does that answers: some rows at once, more of them from the state, then one row after the other."""
    g = gen(12)
    n, d = 150, 72
    f, u = rows(g, n, d, dtype, 0, 0, 2.0, 1.0), rows(g, n, d, dtype)
    w = ref.scan(f.cpu(), u.cpu(), [0, n], None)
    y1, state, _ = ops.gated_scan(f[:70], u[:70], last=True)
    y2, state, _ = ops.gated_scan(f[70:110], u[70:110], None, state, last=True)
    singles = []
    for t in range(110, n):
        singles.append(ops.gated_step(f[t:t + 1], u[t:t + 1], state))
    y = torch.cat([y1, y2] + singles)
    within(y.cpu(), w["h"], w["off"] + U[dtype] * w["h"].abs() + TINY[dtype])
    within(state.cpu(), w["last"], w["off_last"])
