"""Gates of the recurrence that are nearly closed: their smaller share is exp(-|f|) down to the last 32-bit number, and only behind that nothing."""
import math

import pytest
import torch

import sequence_reference as ref
from train_reference import TINY, U, U32, within

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
NAME = {F32: "f32", BF16: "bf16", F16: "f16"}
INF, NAN = float("inf"), float("nan")
# numbers of every type: from 88 on a share has fewer bits than 24, from 150 ln 2 = 103.97 on it is rounded to nothing
OPEN, CLOSED = (80.0, 86.0, 87.0, 88.0, 90.0, 95.0, 100.0, 103.0), (105.0, 120.0)
GATES = [s * f for f in OPEN + CLOSED for s in (1.0, -1.0)]
D = len(GATES)
IS_OPEN = torch.tensor([abs(f) < 104 for f in GATES])
FORGETS = torch.tensor([f < -104 for f in GATES])
MASKS = torch.tensor([f > 104 for f in GATES])


@pytest.fixture(scope="module")
def ops():
    import paper_1909_04885_amd as chicle
    return chicle.TrainOps("cuda:0")


def few_bits(f):
    """How far a small share may be off, as `ref.gate_off` has it, and besides by two roundings to steps of 2^-149, by half of one each."""
    f = f.double()
    return (10 + 2 * f.abs().clamp(max=104)) * U32 + 2.0 ** -149 * torch.exp(f.abs().clamp(max=104))


def gates(n, dtype):
    return torch.tensor(GATES).expand(n, D).to(dtype).contiguous()


def case(dtype):
    """Two sequences, one whose state is large before its first row, and one that begins with none, over several tiles; u is zero for some rows."""
    g = torch.Generator().manual_seed(11)
    n, at = 400, [0, 170, 400]
    most = min(1e37, torch.finfo(dtype).max / 8)
    u = ((2 * torch.rand(n, D, generator=g) - 1) * most).to(dtype)
    u[:3] = 0
    u[100:110] = 0
    h0 = torch.zeros(2, D)
    h0[0] = most
    dy = (0.01 * torch.randn(n, D, generator=g)).to(dtype)
    return gates(n, dtype), u, at, h0, dy, torch.randn(2, D, generator=g)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_small_shares_are_worked_out(ops, monkeypatch, dtype, packed):
    print("\ncase small shares", NAME[dtype], packed, flush=True)
    monkeypatch.setattr(ref, "gate_off", few_bits)
    f, u, at, h0, dy, dlast = case(dtype)
    values = given = u.cuda()
    if packed:
        given = ops.pack8(values)
        values = ref.unpack(given.values, given.scales, D)
    values, offsets = values.cpu(), torch.tensor(at, dtype=torch.int32, device="cuda")
    y, last, states = ops.gated_scan(f.cuda(), given, offsets, h0.cuda(), last=True, states=True)
    least = 4 * TINY[F32]                                # states that are so small themselves: products of a row, and of the rows of a wavefront
    w = ref.scan(f, values, at, h0)
    within(last.cpu(), w["last"], w["off_last"] + least, "last")
    within(states.cpu(), w["before"][::ref.KEPT], w["off_before"][::ref.KEPT] + least, "states")
    within(y.cpu(), w["h"], w["off"] + least + U[dtype] * w["h"].abs() + TINY[dtype], "y")
    df, du, dh0 = ops.gated_scan_grad(f.cuda(), given, states, dy.cuda(), offsets, h0.cuda(), dlast.cuda())
    w = ref.scan_grad(f, values, at, h0, dy, dlast)
    within(dh0.cpu(), w["dh0"], w["off_dh0"] + least, "dh0")
    within(du.cpu(), w["du"], w["off_du"] + least, "du")
    within(df.cpu(), w["df"], w["off_df"] + least, "df")
    ops.sync()


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_a_step_with_small_shares(ops, dtype):
    big = min(1e38, torch.finfo(dtype).max)
    pairs = [(1e38, 0.0), (0.0, big), (1e38, -big), (-1e38, 1.0), (1.0, big), (INF, 0.0), (NAN, 0.0), (0.0, INF), (0.0, NAN), (INF, 1.0), (1.0, -INF)]
    x, u = torch.tensor([p[0] for p in pairs])[:, None].expand(-1, D).contiguous(), torch.tensor([p[1] for p in pairs])[:, None].expand(-1, D).to(dtype).contiguous()
    f, state = gates(len(pairs), dtype), x.cuda()
    y = ops.gated_step(f.cuda(), u.cuda(), state)
    a, c, s = ref.gates(f)
    part = [ref.share(a, x.double()), ref.share(c, u.double())]
    want, seen = part[0] + part[1], ref.share(s, x.double().abs()) + ref.share(s, u.double().abs())
    finite = want.isfinite()
    bound = 2 * (few_bits(f) * seen + 2 * U32 * (part[0].abs() + part[1].abs())) + 2 * TINY[F32]
    assert torch.equal(state.cpu().isfinite(), finite)
    within(state.cpu()[finite], want[finite], bound[finite])
    assert torch.equal(y.nan_to_num(7.0), state.to(dtype).nan_to_num(7.0))           # (the state, rounded once)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
@pytest.mark.parametrize("value", [INF, NAN])
def test_what_is_no_number_goes_on_until_a_gate_closes(ops, dtype, packed, value):
    """From one row of u through all later ones, and from one of dy through all earlier ones, over several tiles; a closed gate stops it, or never takes it in."""
    print("\ncase no number", NAME[dtype], packed, value, flush=True)
    g = torch.Generator().manual_seed(3)
    n = 400
    f, u, dy = gates(n, dtype), torch.randn(n, D, generator=g).to(dtype), torch.randn(n, D, generator=g).to(dtype)
    u[5] = value
    given = ops.pack8(u.cuda()) if packed else u.cuda()
    y, last, states = (t.cpu() for t in ops.gated_scan(f.cuda(), given, last=True, states=True))
    assert not y[5:, IS_OPEN].isfinite().any() and not last[0, IS_OPEN].isfinite().any()
    assert bool(y[:5].isfinite().all()) and bool(y[6:, ~IS_OPEN].isfinite().all()) and bool(last[0, ~IS_OPEN].isfinite().all())
    assert bool(y[:, MASKS].eq(0).all()) and not y[5, FORGETS].isfinite().any()
    assert not states[1:, IS_OPEN].isfinite().any() and bool(states[:, ~IS_OPEN].isfinite().all())
    # and from the state before the first row
    h0 = torch.full((1, D), value)
    u[5] = 1.0
    given = ops.pack8(u.cuda()) if packed else u.cuda()
    y, last, _ = (t if t is None else t.cpu() for t in ops.gated_scan(f.cuda(), given, None, h0.cuda(), last=True))
    assert not y[:, IS_OPEN | MASKS].isfinite().any() and bool(y[:, FORGETS].isfinite().all()) and bool(last[0, FORGETS].isfinite().all())
    # gradients
    h0 = torch.ones(1, D).cuda()
    _, _, states = ops.gated_scan(f.cuda(), given, None, h0, states=True)
    dy[300] = value
    df, du, dh0 = (t.cpu() for t in ops.gated_scan_grad(f.cuda(), given, states, dy.cuda(), None, h0, None))
    assert not du[:301, IS_OPEN].isfinite().any() and not df[:301, IS_OPEN].isfinite().any() and not dh0[0, IS_OPEN | MASKS].isfinite().any()
    assert bool(du[301:].isfinite().all()) and bool(df[301:].isfinite().all()) and not du[:, MASKS].any() and not df[:, ~IS_OPEN].any()
    assert bool(du[:300, FORGETS].isfinite().all()) and not du[300, FORGETS].isfinite().any() and not dh0[0, FORGETS].any()


def test_where_a_share_ends(ops):
    """The least share is 2^-149; a gate is closed from where it is rounded to nothing, 150 ln 2, to the exponent's own rounding (2 |f| 2^-24)."""
    edge = 150 * math.log(2)
    f = torch.tensor([[edge - 0.001, edge - 1e-4, edge + 1e-4, edge + 0.001]]).repeat(2, 1)
    f[1] *= -1
    state = torch.tensor([[0.0], [INF]]).repeat(1, 4).cuda()
    u = torch.tensor([[INF], [1.0]]).repeat(1, 4).cuda()
    ops.gated_step(f.cuda(), u, state)
    assert state.isfinite().tolist() == [[False, False, True, True]] * 2
