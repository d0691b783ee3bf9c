"""Root-mean-square norm of rows whose squares are no 32-bit numbers: too large, or, where eps is zero, too small."""
import pytest
import torch

import sequence_reference as ref
from train_reference import TINY, within

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
NAME = {F32: "f32", BF16: "bf16", F16: "f16"}


@pytest.fixture(scope="module")
def ops():
    import paper_1909_04885_amd as chicle
    return chicle.TrainOps("cuda:0")


def case(n, d, dtype, powers, extra=0):
    """Rows of every power of two in turn, some of them with a single value of that size, and gamma around one."""
    g = torch.Generator(device="cuda").manual_seed(n + d)
    x = torch.rand(n, d + extra, generator=g, device="cuda") * 0.9 + 0.1
    x = torch.where(torch.rand(n, d + extra, generator=g, device="cuda") < 0.5, -x, x)
    at = torch.tensor(powers, dtype=torch.float64, device="cuda")[torch.arange(n, device="cuda") % len(powers)]
    x = x.double() * torch.exp2(at)[:, None]
    x[::5, 1:] *= 2.0 ** -6
    gamma = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    most = torch.finfo(dtype).max
    return x.clamp(-most, most).to(dtype)[:, :d], gamma


def bounds(w, gamma, dtype):
    """Of rstd and y: rstd may be a number of fewer bits than 24, off by half of 2^-149 twice, by which y is off for every unit of r gamma."""
    few = TINY[F32]
    return w["off_rstd"] + few, w["off_y"] + few * w["r"].double().abs() * gamma.double().abs(), w["off_y32"] + few * w["r"].double().abs() * gamma.double().abs()


SIZES = [(1, 1, 0), (40, 5, 0), (33, 64, 3), (24, 250, 0), (21, 500, 0), (40, 1000, 1), (14, 1537, 3), (9, 4096, 0), (7, 9001, 0), (8, 20001, 0), (5, 40000, 0)]


@pytest.mark.parametrize("n, d, extra", SIZES)
@pytest.mark.parametrize("dtype", TYPES, ids=NAME.get)
def test_large_values(ops, dtype, n, d, extra):
    """Ordinary rows beside rows of large ones, up to the type's largest: y is of the order of gamma in all of them."""
    print("\ncase large", NAME[dtype], n, d, extra, flush=True)
    x, gamma = case(n, d, dtype, (128, 0, 64, 100, 3, 66, 1) if dtype != F16 else (16, 0, 14, 8), extra)
    if n > 1:
        x[1, d // 2] = torch.finfo(dtype).max           # an ordinary row with one value of these
    for residual in (None, (x.double() * -0.5).to(dtype)):
        w = ref.rms_norm(x, gamma, residual, 1e-5)
        off_rstd, off_y, off_y32 = bounds(w, gamma, dtype)
        y, r, rstd, _ = ops.rms_norm(x, gamma, residual)
        assert torch.equal(r, w["r"])
        within(rstd, w["rstd"], off_rstd, "rstd")
        within(y, w["y"], off_y, "y")
        y8, _, rstd8, kept = ops.rms_norm(x, gamma, residual, y8=True, keep8=True)
        assert torch.equal(rstd8, rstd)
        _, byte = ref.pack(w["y"].abs() + off_y32)
        within(ops.unpack8(y8, F32), w["y"], off_y32 + ref.step_of(byte, d) / 2 + 2.0 ** -23 * w["y"].abs(), "y8")
        dy = torch.randn(n, d, device="cuda").to(dtype)
        b = ref.rms_norm_grad(dy, r, gamma, rstd, None)
        dx, dgamma = ops.rms_norm_grad(dy, r, gamma, rstd)
        within(dx, b["dx"], b["off_dx"] + 2 * TINY[F32], "dx")
        within(dgamma, b["dgamma"], b["off_dgamma"], "dgamma")


@pytest.mark.parametrize("n, d, extra", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAME.get)
def test_small_values_without_eps(ops, dtype, n, d, extra):
    """Down to 2^-120, where one over the root is still a number."""
    print("\ncase small", NAME[dtype], n, d, extra, flush=True)
    x, gamma = case(n, d, dtype, (-110, 0, -60, -90, 3, -75, -50), extra)
    for eps in (0.0, 2.0 ** -140):
        w = ref.rms_norm(x, gamma, None, eps)
        y, _, rstd, _ = ops.rms_norm(x, gamma, eps=eps)
        within(rstd, w["rstd"], w["off_rstd"], "rstd")
        within(y, w["y"], w["off_y"], "y")


@pytest.mark.parametrize("d", [100, 1000, 5000, 20001])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAME.get)
def test_rows_beside_large_ones_are_what_they_are_alone(ops, dtype, d):
    g = torch.Generator(device="cuda").manual_seed(d)
    x, gamma = torch.randn(6, d, generator=g, device="cuda").to(dtype), torch.randn(d, generator=g, device="cuda").to(dtype)
    alone, _, rstd, _ = ops.rms_norm(x, gamma)
    x[2], x[5] = 1e30, float("inf")
    y, _, rstd2, _ = ops.rms_norm(x, gamma)
    others = torch.tensor([0, 1, 3, 4], device="cuda")
    assert torch.equal(y[others], alone[others]) and torch.equal(rstd2[others], rstd[others])
    assert bool(y[2].isfinite().all()) and bool(y[5].isnan().all()) and float(rstd2[5]) == 0.0
