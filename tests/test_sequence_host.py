"""CPU-side checks of the operators of layers over sequences: refusals, workspace sizes, and the definitions that the results are tested against,
these against differences and against plain loops."""
import ctypes
import math

import pytest
import torch

import sequence_reference as ref
import train_reference

EINVAL, ENOMEM = -1, -2
P = ctypes.c_void_p(4096)                                # (never followed: every call here is refused)
ODD = ctypes.c_void_p(4097)
EIGHT = ctypes.c_void_p(4104)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    import paper_1909_04885_amd as m
    return m.load_train_library()


PACK = dict(x=P, ldx=64, n=4, d=64, type=1, q=P, scales=P, ldq=64, stream=None)
UNPACK = dict(q=P, scales=P, ldq=64, n=4, d=64, type=1, out=P, ldo=64, stream=None)
NORM = dict(x=P, ldx=64, residual=P, ldres=64, gamma=P, n=4, d=64, type=1, eps=1e-5, sum=P, ldsum=64, y=P, ldy=64, y_scales=None, sum8=None, sum8_scales=None,
            ldsum8=0, rstd=P, stream=None)
NORM_GRAD = dict(dy=P, lddy=64, sum=P, ldsum=64, sum_scales=None, gamma=P, rstd=P, dsum=P, lddsum=64, n=4, d=64, type=1, dx=P, lddx=64, dgamma=P, ws=P,
                 nbytes=BIG, stream=None)
SCAN = dict(f=P, ldf=64, u=P, ldu=64, u_scales=None, offsets=P, wide=0, sequences=3, h0=P, n=4, d=64, type=1, y=P, ldy=64, last=P, states=P, ws=P, nbytes=BIG,
            flags=None, stream=None)
SCAN_GRAD = dict(f=P, ldf=64, u=P, ldu=64, u_scales=None, offsets=P, wide=0, sequences=3, h0=P, states=P, dy=P, lddy=64, dlast=P, n=4, d=64, type=1, df=P,
                 lddf=64, du=P, lddu=64, dh0=P, ws=P, nbytes=BIG, flags=None, stream=None)
STEP = dict(f=P, ldf=64, u=P, ldu=64, state=P, lds=64, n=4, d=64, type=1, y=P, ldy=64, stream=None)


@pytest.mark.parametrize("name, good, bad, code", [(name, good, bad, code) for name, good, cases in [
    ("chicle_pack8", PACK, [dict(type=3), dict(n=-1), dict(d=0), dict(n=1 << 31), dict(d=1 << 31), dict(ldx=63), dict(ldq=32), dict(ldq=65), dict(ldq=80), dict(x=None),
                            dict(x=ODD), dict(q=None), dict(q=EIGHT), dict(scales=None)]),
    ("chicle_unpack8", UNPACK, [dict(type=-1), dict(n=-1), dict(d=0), dict(ldo=63), dict(ldq=32), dict(ldq=80), dict(q=None), dict(q=ODD), dict(scales=None),
                                dict(out=None), dict(out=ODD)]),
    ("chicle_rms_norm", NORM, [dict(type=9), dict(n=-1), dict(d=0), dict(ldx=63), dict(ldres=1), dict(ldsum=63), dict(ldy=63), dict(eps=-1.0),
                               dict(eps=float("nan")), dict(x=None), dict(x=ODD), dict(residual=ODD), dict(gamma=None), dict(sum=ODD), dict(y=None), dict(rstd=None),
                               dict(rstd=ODD), dict(y_scales=P, ldy=80), dict(y_scales=P, y=EIGHT), dict(sum8=P, sum8_scales=None, ldsum8=64),
                               dict(sum8=P, sum8_scales=P, ldsum8=32)]),
    ("chicle_rms_norm_grad", NORM_GRAD, [dict(type=9), dict(n=-1), dict(d=0), dict(lddy=63), dict(ldsum=63), dict(lddsum=63), dict(lddx=63), dict(dy=None),
                                         dict(sum=None), dict(sum=ODD), dict(sum_scales=P, ldsum=80), dict(sum_scales=P, sum=EIGHT), dict(gamma=None),
                                         dict(rstd=None), dict(dsum=ODD), dict(dx=None), dict(dgamma=None), dict(ws=ODD)]),
    ("chicle_gated_scan", SCAN, [dict(type=9), dict(n=-1), dict(d=0), dict(n=1 << 31), dict(ldf=63), dict(ldu=63), dict(ldy=63), dict(sequences=-1),
                                 dict(sequences=1 << 31), dict(offsets=None), dict(offsets=None, sequences=0), dict(offsets=ODD), dict(offsets=ctypes.c_void_p(4100), wide=1),
                                 dict(h0=ODD), dict(f=None), dict(u=None), dict(u=ODD), dict(u_scales=P, ldu=80), dict(u_scales=P, u=EIGHT), dict(y=None),
                                 dict(last=ODD), dict(states=ODD), dict(ws=ODD)]),
    ("chicle_gated_scan_grad", SCAN_GRAD, [dict(type=9), dict(n=-1), dict(d=0), dict(ldf=63), dict(ldu=63), dict(lddy=63), dict(lddf=63), dict(lddu=63),
                                           dict(sequences=-1), dict(offsets=None), dict(states=None), dict(states=ODD), dict(dy=None), dict(df=None), dict(du=ODD),
                                           dict(dlast=ODD), dict(dh0=ODD), dict(h0=ODD), dict(u_scales=P, ldu=96, d=97, ldf=97, lddy=97, lddf=97, lddu=97),
                                           dict(ws=ODD)]),
    ("chicle_gated_step", STEP, [dict(type=9), dict(n=-1), dict(d=0), dict(ldf=63), dict(ldu=63), dict(lds=63), dict(ldy=63), dict(f=None), dict(u=ODD),
                                 dict(state=None), dict(state=ODD), dict(y=None)])] for bad in cases for code in [EINVAL]] + [
    ("chicle_rms_norm_grad", NORM_GRAD, dict(nbytes=8), ENOMEM), ("chicle_gated_scan", SCAN, dict(nbytes=8), ENOMEM),
    ("chicle_gated_scan_grad", SCAN_GRAD, dict(nbytes=8), ENOMEM)])
def test_refusals(lib, name, good, bad, code):
    args = dict(good, **bad)
    assert set(args) == set(good)
    assert getattr(lib, name)(*args.values()) == code
    assert lib.chicle_train_last_error()


# (four rows of 64 columns: 128 bytes of f, u and y, 256 of the state)
@pytest.mark.parametrize("name", ["f", "u", "y"])
@pytest.mark.parametrize("place", [
    dict(), dict(at=4096 + 896), dict(at=4096 - 510), dict(at=4096 + 128, ld=128), dict(at=4096 + 254, ld=192, lds=96), dict(at=4096 + 258, ld=192, lds=96),
    dict(at=4096 - 130, ld=192, lds=96, n=2), dict(at=4096 - 126 - 384, ld=192, lds=96), dict(at=4096, ld=64, n=1), dict(at=4096 + 256, ld=256, lds=96)])
def test_a_state_that_another_tensor_overlaps_is_refused(lib, name, place):
    ld, state = place.get("ld", 64), 4096
    args = dict(STEP, f=ctypes.c_void_p(1 << 20), u=ctypes.c_void_p(1 << 21), y=ctypes.c_void_p(1 << 22), state=P, n=place.get("n", 4), lds=place.get("lds", 64))
    args.update({name: ctypes.c_void_p(place.get("at", state)), "ld" + name: ld})
    assert lib.chicle_gated_step(*args.values()) == EINVAL and b"overlap" in lib.chicle_train_last_error()


def test_workspace_sizes(lib):
    assert lib.chicle_rms_norm_grad_bytes(-1, 4, 0) == 0 and lib.chicle_rms_norm_grad_bytes(4, 0, 0) == 0 and lib.chicle_rms_norm_grad_bytes(4, 4, 7) == 0
    assert lib.chicle_gated_scan_bytes(-1, 4, 0) == 0 and lib.chicle_gated_scan_bytes(4, 0, 0) == 0 and lib.chicle_gated_scan_bytes(4, 4, 3) == 0
    assert 0 < lib.chicle_rms_norm_grad_bytes(0, 64, 0) and 0 < lib.chicle_gated_scan_bytes(0, 64, 0)
    assert lib.chicle_gated_scan_bytes(65536, 2048, 1) < 65536 * 2048              # less than a byte for a value


@pytest.mark.parametrize("rows, whole", [(0, True), (6, True), (7, False), (5, False)])
def test_rows_that_are_no_whole_sequences_are_refused(rows, whole):
    from paper_1909_04885_amd.local_sgd import SequenceModel
    model = SequenceModel(8, 4, 16, 1, 3, torch.float32, "cpu")
    if whole:
        assert model.offsets(rows, "cpu").tolist() == list(range(0, rows + 1, 3))
    else:
        with pytest.raises(ValueError):
            model.offsets(rows, "cpu")


@pytest.mark.parametrize("n, d", [(1 << 30, 64), ((1 << 30) - 127, 1), (129, (1 << 28) - 63), (1 << 20, 1 << 16)])
def test_scans_of_more_workgroups_than_a_launch_has_are_refused(lib, n, d):
    big = dict(n=n, d=d, ldf=d, ldu=d, ldy=d)
    assert lib.chicle_gated_scan(*dict(SCAN, **big).values()) == EINVAL and b"too many" in lib.chicle_train_last_error()
    big = dict(n=n, d=d, ldf=d, ldu=d, lddy=d, lddf=d, lddu=d)
    assert lib.chicle_gated_scan_grad(*dict(SCAN_GRAD, **big).values()) == EINVAL and b"too many" in lib.chicle_train_last_error()


def test_reference_of_the_8_bits():
    """The scale is the least power of two that is enough, and values come back to half of it."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn(40, 70, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-130, 100, (40, 1), generator=g).double())
    q, byte = ref.pack(x)
    step = ref.step_of(byte, 70)
    top = torch.nn.functional.pad(x, (0, 26)).view(40, 3, 32).abs().amax(2)
    power = torch.exp2(byte.double() - 127)
    assert bool((top <= 127 * power).all()) and bool(((top > 127 * power / 2) | (byte == 1)).all())
    assert float(q.abs().max()) <= 127 and not q[:, 70:].any()
    assert bool(((ref.unpack(q, byte, 70) - x).abs() <= step / 2).all())


def test_reference_scan_against_a_plain_loop():
    g = torch.Generator().manual_seed(5)
    f, u, h0 = torch.randn(9, 3, generator=g), torch.randn(9, 3, generator=g), torch.randn(3, 3, generator=g)
    r = ref.scan(f, u, [1, 4, 4, 8], h0)
    for c in range(3):
        for j, (lo, hi) in enumerate([(1, 4), (4, 4), (4, 8)]):
            h = float(h0[j, c])
            for t in range(lo, hi):
                a = 1 / (1 + math.exp(-float(f[t, c])))
                assert abs(float(r["before"][t, c]) - h) < 1e-14
                h = a * h + (1 - a) * float(u[t, c])
                assert abs(float(r["h"][t, c]) - h) < 1e-14
            assert abs(float(r["last"][j, c]) - h) < 1e-14
    assert not r["h"][0].any() and not r["h"][8].any()


def test_reference_gradients_against_differences():
    """Central differences in 64 bits: off by h^2 times a third derivative of order one, and 2^-52 / h."""
    g = torch.Generator().manual_seed(1)
    eps, tol, f64 = 1e-5, 1e-8, torch.float64
    n, d, at = 12, 4, [0, 5, 5, 11]
    f, u, dy = (torch.randn(n, d, dtype=f64, generator=g) for _ in range(3))
    h0, dlast = torch.randn(3, d, dtype=f64, generator=g), torch.randn(3, d, dtype=f64, generator=g)
    gamma, dr = torch.randn(d, dtype=f64, generator=g), torch.randn(n, d, dtype=f64, generator=g)

    def scanned(f, u, h0):
        r = ref.scan(f, u, at, h0)
        return float((r["h"] * dy).sum() + (r["last"] * dlast).sum())

    def normed(x, gamma):
        return float((ref.rms_norm(x, gamma, None, 1e-5)["y"] * dy).sum() + (x * dr).sum())

    train_reference.U[f64], train_reference.TINY[f64] = 2.0 ** -53, 0.0
    try:
        r = ref.scan_grad(f, u, at, h0, dy, dlast)
        b = ref.rms_norm_grad(dy, u, gamma, ref.rms_norm(u, gamma, None, 1e-5)["rstd"], dr)
        for _ in range(5):
            v, w, z = torch.randn(n, d, dtype=f64, generator=g), torch.randn(3, d, dtype=f64, generator=g), torch.randn(d, dtype=f64, generator=g)
            for got, what, moved in ((r["df"], v, lambda s: scanned(f + s * v, u, h0)), (r["du"], v, lambda s: scanned(f, u + s * v, h0)),
                                     (r["dh0"], w, lambda s: scanned(f, u, h0 + s * w)), (b["dx"], v, lambda s: normed(u + s * v, gamma)),
                                     (b["dgamma"], z, lambda s: normed(u, gamma + s * z))):
                assert abs((moved(eps) - moved(-eps)) / (2 * eps) - float((got * what).sum())) < tol
    finally:
        del train_reference.U[f64], train_reference.TINY[f64]


def test_no_kernel_keeps_registers_in_scratch_memory(lib):
    """The kernels' metadata in the library that was built here, those of every source file."""
    import struct

    import msgpack

    import paper_1909_04885_amd as m
    data, at, kernels, bundles = open(m.train_library_path(), "rb").read(), -1, [], 0
    while (at := data.find(b"__CLANG_OFFLOAD_BUNDLE__", at + 1)) >= 0:
        count, pos = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for _ in range(count):
            offset, size, name = struct.unpack_from("<3Q", data, pos)
            if b"gfx950" in data[pos + 24:pos + 24 + name]:
                kernels += metadata(data[at + offset:at + offset + size], struct, msgpack)
                bundles += 1
            pos += 24 + name
    assert bundles == 2 and len(kernels) > 100
    assert any("scan_backward" in k[".name"] for k in kernels)
    assert [k[".name"] for k in kernels if k[".private_segment_fixed_size"] > 0] == []


def metadata(elf, struct, msgpack):
    sections, entry, number = struct.unpack_from("<Q", elf, 40)[0], *struct.unpack_from("<2H", elf, 58)
    kernels = []
    for i in range(number):
        kind, offset, size = struct.unpack_from("<I", elf, sections + i * entry + 4)[0], *struct.unpack_from("<2Q", elf, sections + i * entry + 24)
        while kind == 7 and size > 0:
            name, desc, what = struct.unpack_from("<3I", elf, offset)
            start = offset + 12 + (name + 3) // 4 * 4
            if what == 32 and elf[offset + 12:offset + 18] == b"AMDGPU":
                kernels += msgpack.unpackb(elf[start:start + desc])["amdhsa.kernels"]
            size -= start + (desc + 3) // 4 * 4 - offset
            offset = start + (desc + 3) // 4 * 4
    return kernels
