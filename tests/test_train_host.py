"""CPU-side checks of the training operators' library: exported symbols, refusals, workspace sizes, and the definitions that the
results are tested against, these against differences."""
import ctypes
import os
import re

import pytest
import torch

import train_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ENOMEM = -1, -2
P = ctypes.c_void_p(4096)                                # (never followed: every call here is refused)
ODD = ctypes.c_void_p(4097)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    import paper_1909_04885_amd as m
    return m.load_train_library()


def test_library_exports_every_declared_symbol(lib):
    from paper_1909_04885_amd.train import TRAIN_EXPORTS
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "chicle_train.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(chicle_[a-z_0-9]+)\s*\(", text)))
    assert sorted(TRAIN_EXPORTS) == names
    for n in names:
        assert hasattr(lib, n), n


def test_no_gpu_is_an_error_and_not_another_path():
    if torch.cuda.is_available():
        pytest.skip("a GPU is here")
    import paper_1909_04885_amd as m
    with pytest.raises(m.ChicleError):
        m.TrainOps()


LOSS = dict(x=P, ldx=64, w=P, ldw=64, labels=P, wide=0, n=4, d=64, classes=10, type=1, loss=P, lse=P, ws=P, nbytes=BIG, flags=None, stream=None)
GRAD = dict(x=P, ldx=64, w=P, ldw=64, labels=P, wide=0, rw=P, n=4, d=64, classes=10, type=1, loss=P, dx=P, lddx=64, dw=P, lddw=64, ws=P, nbytes=BIG,
            flags=None, stream=None)
EMBED = dict(table=P, ld=64, rows=10, ids=P, wide=0, n=4, d=64, type=0, scale=1.0, out=P, ldo=64, flags=None, stream=None)
EMBED_GRAD = dict(ids=P, wide=0, dout=P, ldd=64, n=4, d=64, rows=10, type=0, scale=1.0, accumulate=0, out=P, ldo=64, ws=P, nbytes=BIG, flags=None,
                  stream=None)
NORM = dict(x=P, ldx=64, gamma=P, beta=P, n=4, d=64, type=0, eps=1e-5, y=P, ldy=64, mean=P, rstd=P, stream=None)
NORM_GRAD = dict(dy=P, lddy=64, x=P, ldx=64, gamma=P, mean=P, rstd=P, n=4, d=64, type=0, dx=P, lddx=64, dgamma=P, dbeta=P, ws=P, nbytes=BIG, stream=None)


@pytest.mark.parametrize("name, good, bad, code", [
    ("chicle_softmax_loss", LOSS, bad, code) for bad, code in [
        (dict(type=3), EINVAL), (dict(n=-1), EINVAL), (dict(d=0), EINVAL), (dict(classes=0), EINVAL), (dict(ldx=63), EINVAL), (dict(ldw=63), EINVAL),
        (dict(x=None), EINVAL), (dict(w=None), EINVAL), (dict(labels=None), EINVAL), (dict(loss=None), EINVAL), (dict(lse=ODD), EINVAL),
        (dict(x=ODD), EINVAL), (dict(n=1 << 22), EINVAL), (dict(classes=1 << 30), EINVAL), (dict(n=1 << 21, classes=1 << 29), EINVAL),
        (dict(nbytes=16), ENOMEM), (dict(ws=ODD), EINVAL)]] + [
    ("chicle_softmax_loss_grad", GRAD, bad, code) for bad, code in [
        (dict(type=-1), EINVAL), (dict(lddx=63), EINVAL), (dict(lddw=1), EINVAL), (dict(dw=None), EINVAL), (dict(dx=None), EINVAL), (dict(rw=None), EINVAL),
        (dict(rw=ODD), EINVAL), (dict(nbytes=0), ENOMEM)]] + [
    ("chicle_embed", EMBED, bad, code) for bad, code in [
        (dict(type=7), EINVAL), (dict(n=-1), EINVAL), (dict(d=0), EINVAL), (dict(rows=0), EINVAL), (dict(ld=63), EINVAL), (dict(ldo=63), EINVAL),
        (dict(table=None), EINVAL), (dict(ids=None), EINVAL), (dict(out=ODD), EINVAL), (dict(d=1 << 23, ld=1 << 23, ldo=1 << 23), EINVAL)]] + [
    ("chicle_embed_grad", EMBED_GRAD, bad, code) for bad, code in [
        (dict(type=7), EINVAL), (dict(n=-1), EINVAL), (dict(rows=(1 << 31) - 1), EINVAL), (dict(ldd=63), EINVAL), (dict(dout=None), EINVAL),
        (dict(out=None), EINVAL), (dict(nbytes=64), ENOMEM)]] + [
    ("chicle_layer_norm", NORM, bad, code) for bad, code in [
        (dict(type=7), EINVAL), (dict(n=-1), EINVAL), (dict(d=0), EINVAL), (dict(ldx=63), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL),
        (dict(gamma=None), EINVAL), (dict(mean=ODD), EINVAL)]] + [
    ("chicle_layer_norm_grad", NORM_GRAD, bad, code) for bad, code in [
        (dict(type=7), EINVAL), (dict(n=-1), EINVAL), (dict(lddx=63), EINVAL), (dict(dgamma=None), EINVAL), (dict(dy=None), EINVAL), (dict(nbytes=8), ENOMEM)]])
def test_refusals(lib, name, good, bad, code):
    args = dict(good, **bad)
    assert getattr(lib, name)(*args.values()) == code
    assert lib.chicle_train_last_error()


def test_clip_refusals(lib):
    ins, sizes = (ctypes.c_void_p * 2)(4096, 8192), (ctypes.c_int64 * 2)(10, 10)
    types = (ctypes.c_int32 * 2)(0, 1)
    call = lambda **k: lib.chicle_clip_grads(*dict(dict(i=ins, o=ins, s=sizes, t=types, n=2, m=1.0, norm=P, ws=P, nb=BIG, st=None), **k).values())  # noqa: E731
    assert call(n=-1) == EINVAL and call(i=None) == EINVAL and call(norm=None) == EINVAL and call(m=-1.0) == EINVAL and call(m=float("nan")) == EINVAL
    assert call(t=(ctypes.c_int32 * 2)(0, 9)) == EINVAL and call(s=(ctypes.c_int64 * 2)(10, -1)) == EINVAL
    assert call(i=(ctypes.c_void_p * 2)(4096, None)) == EINVAL and call(i=(ctypes.c_void_p * 2)(4098, 8192)) == EINVAL
    assert call(s=(ctypes.c_int64 * 2)(1 << 60, 1)) == EINVAL
    assert call(nb=0) == ENOMEM


def test_workspace_sizes(lib):
    size = lib.chicle_softmax_loss_bytes
    assert size(256, 64, 256, 64, 4, 64, 10, 9, 0) == 0 and size(256, 64, 256, 64, -1, 64, 10, 1, 0) == 0
    one, many = size(256, 1024, 256, 1024, 1, 1024, 32000, 1, 0), size(256, 2048, 256, 2048, 8192, 2048, 128000, 1, 1)
    assert one < 1 << 20                                 # rows that can be read where they are are not copied
    assert many < 8192 * 128000 * 2                      # less than the logits would take, in 16 bits
    assert 0 < size(None, 64, 256, 64, 0, 64, 10, 1, 1) <= 4096 and 0 < lib.chicle_embed_grad_bytes(0, 64, 10) and 0 < lib.chicle_layer_norm_grad_bytes(0, 64, 0)
    assert lib.chicle_embed_grad_bytes(-1, 4, 4) == 0 and lib.chicle_layer_norm_grad_bytes(4, 0, 0) == 0
    assert 0 < lib.chicle_embed_grad_bytes(1000, 64, 50) < lib.chicle_embed_grad_bytes(100000, 64, 50)


def test_reference_gradients_against_differences():
    """Central differences in 64 bits: off by h^2 times a third derivative of order one, and 2^-52 / h."""
    g = torch.Generator().manual_seed(1)
    h, tol = 1e-5, 1e-8
    x, w = torch.randn(6, 5, dtype=torch.float64, generator=g), torch.randn(9, 5, dtype=torch.float64, generator=g)
    labels, weight = torch.tensor([0, 8, -1, 3, 3, 1]), torch.rand(6, dtype=torch.float64, generator=g)

    def total(x, w):
        lse = torch.logsumexp(x @ w.t(), 1)
        z = (x @ w.t())[torch.arange(6), labels.clamp(min=0)]
        return float((weight * (lse - z))[labels >= 0].sum())

    ref.U[torch.float64], ref.TINY[torch.float64] = 2.0 ** -53, 0.0
    try:
        r = ref.softmax_loss(x, w, labels, weight)
        gamma, beta = torch.randn(5, dtype=torch.float64, generator=g), torch.randn(5, dtype=torch.float64, generator=g)
        dy = torch.randn(6, 5, dtype=torch.float64, generator=g)
        f = ref.layer_norm(x, gamma, beta, 1e-5)
        b = ref.layer_norm_grad(dy, x, gamma, f["mean"], f["rstd"])

        def normed(x, gamma, beta):
            return float((dy * ref.layer_norm(x, gamma, beta, 1e-5)["y"]).sum())

        for _ in range(5):
            v, u = torch.randn(6, 5, dtype=torch.float64, generator=g), torch.randn(9, 5, dtype=torch.float64, generator=g)
            q = torch.randn(5, dtype=torch.float64, generator=g)
            assert abs((total(x + h * v, w) - total(x - h * v, w)) / (2 * h) - float((r["dx"] * v).sum())) < tol
            assert abs((total(x, w + h * u) - total(x, w - h * u)) / (2 * h) - float((r["dw"] * u).sum())) < tol
            assert abs((normed(x + h * v, gamma, beta) - normed(x - h * v, gamma, beta)) / (2 * h) - float((b["dx"] * v).sum())) < tol
            assert abs((normed(x, gamma + h * q, beta) - normed(x, gamma - h * q, beta)) / (2 * h) - float((b["dgamma"] * q).sum())) < tol
            assert abs((normed(x, gamma, beta + h * q) - normed(x, gamma, beta - h * q)) / (2 * h) - float((b["dbeta"] * q).sum())) < tol
    finally:
        del ref.U[torch.float64], ref.TINY[torch.float64]


def test_no_kernel_keeps_registers_in_scratch_memory(lib):
    """The kernels' metadata in the library that was built here."""
    import struct
    import msgpack
    import paper_1909_04885_amd as m
    data = open(m.train_library_path(), "rb").read()
    at = data.index(b"__CLANG_OFFLOAD_BUNDLE__")
    count, pos, elf = struct.unpack_from("<Q", data, at + 24)[0], at + 32, None
    for _ in range(count):
        offset, size, name = struct.unpack_from("<3Q", data, pos)
        if b"gfx950" in data[pos + 24:pos + 24 + name]:
            elf = data[at + offset:at + offset + size]
        pos += 24 + name
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
    assert len(kernels) > 20
    assert [k[".name"] for k in kernels if k[".private_segment_fixed_size"] > 0] == []
