"""CPU-side checks of what the training operators ask for: memory in proportion to the data."""
import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_1909_04885_amd as m
    return m.load_train_library()


@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("d", [250, 1024, 4096])
def test_workspace_of_the_losss_gradient_grows_with_the_rows_and_not_faster(lib, kind, d):
    classes, rows = 128000, [32768, 65536, 131072, 262144, 1 << 20]
    size = [lib.chicle_softmax_loss_bytes(4096, d, 4096, d, n, d, classes, kind, 1) for n in rows]
    for n, s in zip(rows, size):
        # x and w laid out, dx in 32 bits, two planes of a gigabyte or of min(8 d, 2^24 / d) classes, a maximum and a sum of every row and half a tile of 256 classes
        wide = (d + 127) // 64 * 64
        assert s <= 2 * (n + classes) * wide + 4 * n * wide + max(4 * n * min(8 * d, (1 << 24) // d), 1 << 30) + n * (classes // 256) * 2 * 8 + (1 << 28), n
        assert s < 2 * n * classes                       # less than the logits would take


def test_refusals_of_taking_flags(lib):
    import ctypes
    p, odd = ctypes.c_void_p(4096), ctypes.c_void_p(4098)
    for flags, out in ((None, p), (p, None), (odd, p), (p, odd)):
        assert lib.chicle_train_take_flags(flags, out, None) == -1


def test_outputs_of_clipping_that_overlap_are_refused(lib):
    import ctypes
    ins, sizes, types = (ctypes.c_void_p * 3)(4096, 8192, 16384), (ctypes.c_int64 * 3)(10, 100, 10), (ctypes.c_int32 * 3)(0, 1, 0)
    norm, ws = ctypes.c_void_p(4096), ctypes.c_void_p(4096)
    for out in ((4096, 8192, 4096), (16384, 4096, 4292), (8188, 8192, 4096), (4096, 4132, 9000)):
        assert lib.chicle_clip_grads(ins, (ctypes.c_void_p * 3)(*out), sizes, types, 3, 1.0, norm, ws, 1 << 40, None) == -1, out
        assert b"twice" in lib.chicle_train_last_error()
    # side by side, and one of no values beside another: these get as far as the workspace
    for out, many in (((4096, 8192, 4136), (10, 100, 10)), ((8192, 8192, 4096), (10, 0, 10))):
        assert lib.chicle_clip_grads(ins, (ctypes.c_void_p * 3)(*out), (ctypes.c_int64 * 3)(*many), types, 3, 1.0, norm, ws, 0, None) == -2
