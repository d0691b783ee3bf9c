"""Recurrences that remember for thousands of rows, over many tiles, groups and runs of them, against their definition in 64 bits."""
import pytest
import torch

import sequence_cases as cases
import sequence_reference as ref
from train_reference import TINY, U, U32, within

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
NAME = {F32: "f32", BF16: "bf16", F16: "f16"}
INF = float("inf")


@pytest.fixture(scope="module")
def ops():
    import paper_1909_04885_amd as chicle
    return chicle.TrainOps("cuda:0")


@pytest.mark.parametrize("kind, d, dtype, packed", [("one", 130, F32, False), ("one", 130, BF16, True), ("one", 3, F16, False), ("some", 3, F32, True), ("some", 3, BF16, False),
                                                    ("some", 130, F16, True)], ids=lambda x: NAME.get(x, str(x)))
def test_states_that_last(ops, kind, d, dtype, packed):
    print("\ncase states that last", kind, d, NAME[dtype], packed, flush=True)
    f, u, at, h0, dy, dlast = cases.long_memory(kind, d, dtype)
    given = u.cuda()
    if packed:
        given = ops.pack8(given)
        u = ref.unpack(given.values, given.scales, d).cpu()
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    y, last, states = ops.gated_scan(f.cuda(), given, offsets, h0.cuda(), last=True, states=True)
    df, du, dh0 = ops.gated_scan_grad(f.cuda(), given, states, dy.cuda(), offsets, h0.cuda(), dlast.cuda())
    ops.sync()
    w = ref.scan(f, u, at, h0)
    within(y.cpu(), w["h"], w["off"] + U[dtype] * w["h"].abs() + TINY[dtype], "y")
    within(last.cpu(), w["last"], w["off_last"], "last")
    within(states.cpu(), w["before"][::ref.KEPT], w["off_before"][::ref.KEPT], "states")
    w = ref.scan_grad(f, u, at, h0, dy, dlast)
    within(dh0.cpu(), w["dh0"], w["off_dh0"], "dh0")
    within(du.cpu(), w["du"], w["off_du"], "du")
    within(df.cpu(), w["df"], w["off_df"], "df")


@pytest.mark.parametrize("n", [129, 1025, 8193, 70000])
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_a_state_goes_through_masked_rows_as_it_is(ops, dtype, n):
    """Every row masked: the state before the first row is there after the last one, bit for bit, and the last one's gradient is the first one's."""
    g = torch.Generator(device="cuda").manual_seed(n)
    for d in (3, 130):
        f, u = torch.full((n, d), INF, dtype=dtype, device="cuda"), torch.full((n, d), float("nan"), dtype=dtype, device="cuda")
        h0, dlast = torch.randn(1, d, generator=g, device="cuda"), torch.randn(1, d, generator=g, device="cuda")
        y, last, states = ops.gated_scan(f, u, None, h0, last=True, states=True)
        assert torch.equal(last, h0) and torch.equal(states, h0.expand(len(states), d)) and torch.equal(y, h0.to(dtype).expand(n, d))
        df, du, dh0 = ops.gated_scan_grad(f, u, states, torch.zeros_like(f), None, h0, dlast)
        assert torch.equal(dh0, dlast) and not df.any() and not du.any()


@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_a_row_is_seen_through_masked_ones(ops, dtype):
    """One row that is not masked, at the beginning of a run of tiles, inside it and at its end: what it takes in stays, what reaches it comes from the end."""
    n, d = 30000, 66
    near = 32 * U32                                      # (a gate's share at 0: ten roundings, and its use)
    for row in (0, 127, 128, 8191, 8192, 9000, 16384 + 1023, 29999):
        f, u, dy = torch.full((n, d), INF, dtype=dtype, device="cuda"), torch.zeros(n, d, dtype=dtype, device="cuda"), torch.zeros(n, d, dtype=dtype, device="cuda")
        f[row], u[row] = 0.0, 2.0                        # half of the state and half of u: 0.5 and 1
        h0, dlast = torch.ones(1, d, device="cuda"), torch.full((1, d), 4.0, device="cuda")
        y, last, states = ops.gated_scan(f, u, None, h0, last=True, states=True)
        want = torch.full((n, d), 1.5, device="cuda")
        want[:row] = 1.0
        within(last, want[-1:], 1.5 * near, "last")
        within(y, want, 1.5 * (near + U[dtype]), "y")
        df, du, dh0 = ops.gated_scan_grad(f, u, states, dy, None, h0, dlast)
        within(dh0, 0.5 * dlast, 2 * near, "dh0")
        within(du[row], 0.5 * dlast[0], 2 * (near + U[dtype]), "du")
        within(df[row], -0.25 * dlast[0], near + U[dtype], "df")         # G (h - u) a (1 - a)
        du[row] = df[row] = 0
        assert not du.any() and not df.any()
