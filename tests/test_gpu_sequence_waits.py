"""A scan whose tiles give up waiting for one another says so: the bounded wait is given no time from here, so that every kernel ends as it always does."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_wait_that_is_given_up_is_reported(dtype):
    import paper_1909_04885_amd as chicle
    ops, looks = chicle.TrainOps("cuda:0"), ctypes.c_int32.in_dll(chicle.load_train_library(), "chicle_scan_looks")
    g = torch.Generator(device="cuda").manual_seed(1)
    f, u, dy = (torch.randn(65536, 64, generator=g, device="cuda").to(dtype) for _ in range(3))    # (512 tiles that begin together, one after the other's state)
    y, last, states = ops.gated_scan(f, u, last=True, states=True)
    df, du, _ = ops.gated_scan_grad(f, u, states, dy)
    ops.sync()
    usual = looks.value
    assert usual == 1 << 22
    try:
        looks.value = 0
        for call in (lambda: ops.gated_scan(f, u), lambda: ops.gated_scan_grad(f, u, states, dy)):
            call()
            with pytest.raises(chicle.ChicleError, match="waited"):
                ops.sync()
            ops.sync()                                   # (once)
        wrong = torch.tensor([0, 70000], dtype=torch.int32, device="cuda")
        ops.gated_scan(f, u, wrong)
        with pytest.raises(chicle.ChicleError, match="offset.*waited"):
            ops.sync()
    finally:
        looks.value = usual
    again = ops.gated_scan(f, u, last=True, states=True) + ops.gated_scan_grad(f, u, states, dy)[:2]
    assert all(torch.equal(p, q) for p, q in zip(again, (y, last, states, df, du)))
    ops.sync()
