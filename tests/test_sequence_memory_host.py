"""What the tests of recurrences with a long memory would see: a state that is lost between tiles, groups or runs is far outside of the bounds.  (Mistakes are made
here in the oracle, by beginning anew where the state should have gone on.)"""
import pytest
import torch

import sequence_cases as cases
import sequence_reference as ref


@pytest.fixture(scope="module")
def right():
    f, u, at, h0, dy, dlast = cases.long_memory("one", 3, torch.float32)
    return f, u, h0, ref.scan(f, u, at, h0)


@pytest.mark.parametrize("lost", [128, 8 * 128, 64 * 128, 128 * 128])
def test_a_state_that_is_lost_shows(right, lost):
    f, u, h0, w = right
    wrong = ref.scan(f[lost:], u[lost:], [0, cases.ROWS - lost], None)
    off = (wrong["h"] - w["h"][lost:]).abs()
    assert bool((off[:100] > 3 * w["off"][lost:][:100])[:, 1:].all())
    assert float(w["off"].max()) < 0.05                  # (of states around one)


@pytest.mark.parametrize("tiles", [1, 8, 64])
def test_a_share_that_is_left_out_shows(right, tiles):
    """The product of the shares of so many tiles, taken as one."""
    f, u, h0, w = right
    a = ref.gates(f)[0]
    at = 64 * 128
    missing = a[at - 128 * tiles:at].log().sum(0).exp()
    off = w["h"][at - 128 * tiles - 1].abs() * (1 - missing)
    assert int((off > 3 * w["off"][at]).sum()) >= 2
