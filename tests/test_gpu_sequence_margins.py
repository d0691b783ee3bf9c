"""What the scan and its gradients write lies inside of their outputs and their workspace, whatever the offsets are: through the C ABI, with all of them in one
buffer, known bytes between them, and rows with known bytes behind them."""
import pytest
import torch

import sequence_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAME = {F32: "f32", BF16: "bf16", F16: "f16"}
TYPE = {F32: 0, BF16: 1, F16: 2}
MARGIN, FILL = 4096, 0xA5
N, D = 3000, 70                                          # 24 tiles, three groups of them, and two column blocks; a last tile that is not full

RIGHT = [[0, 3000], [0, 1000, 1000, 1029, 3000], [130, 257, 2900]]
WRONG = [[0, 1500, 1400, 3000], [0, 128, 127, 129, 3000], [0, 2048, 1023, 3000], list(range(3000, -1, -50)), [3000, 0], [2999, 3000, 2999], [0, 3001], [0, 2900, 5000],
         [-7, 500, 3000], [0, 2 ** 31 - 1, 100, 3000], [-2 ** 31, 2 ** 31 - 1], [5000, 6000], [0, -1, -1, 3000], [0, 1000, 1000, 999, 1000, 3000]]
WRONG_WIDE = [[0, 2 ** 32 + 5, 3000], [-2 ** 40, 10, 3000], [0, 2 ** 63 - 1, 2 ** 63 - 1], [2 ** 32, 2 ** 32 + 3000], [0, 1500, -2 ** 63, 3000]]


class Buffer:
    """Parts of one allocation with margins before, between and behind them."""

    def __init__(self, **sizes):
        self.at, end = {}, MARGIN
        for name, size in sizes.items():
            self.at[name] = (end, size)
            end = (end + size + MARGIN + 255) // 256 * 256
        self.bytes = torch.full((end,), FILL, dtype=torch.uint8, device="cuda")

    def pointer(self, name):
        return self.bytes.data_ptr() + self.at[name][0]

    def part(self, name, dtype, shape):
        begin, size = self.at[name]
        return self.bytes[begin:begin + size].view(dtype).view(shape)

    def margins_are_whole(self, ld, d, size, rows):
        inside = torch.zeros_like(self.bytes, dtype=torch.bool)
        for begin, length in self.at.values():
            inside[begin:begin + length] = True
        for name in rows:                                # (what lies between two rows is a margin, too)
            begin, length = self.at[name]
            inside[begin:begin + length].view(-1, ld * size)[:, d * size:] = False
        return bool((self.bytes[~inside] == FILL).all())


@pytest.mark.parametrize("wide, at, wrong", [(False, x, False) for x in RIGHT] + [(True, x, False) for x in RIGHT[1:]] + [(False, x, True) for x in WRONG] +
                         [(True, x, True) for x in WRONG + WRONG_WIDE])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAME.get)
def test_nothing_is_written_beside_the_outputs(dtype, wide, at, wrong):
    import paper_1909_04885_amd as chicle
    print("\ncase margins", NAME[dtype], wide, at[:6], flush=True)
    ops, lib = chicle.TrainOps("cuda:0"), chicle.load_train_library()
    g = torch.Generator(device="cuda").manual_seed(7)
    k, size, ld = len(at) - 1, torch.finfo(dtype).bits // 8, D + 6
    f, u, dy = (torch.randn(N, D, generator=g, device="cuda").to(dtype) for _ in range(3))
    h0, dlast = torch.randn(k, D, generator=g, device="cuda"), torch.randn(k, D, generator=g, device="cuda")
    offsets = torch.tensor(at, dtype=torch.int64 if wide else torch.int32, device="cuda")
    kept = -(-N // ref.KEPT)
    nbytes = lib.chicle_gated_scan_bytes(N, D, TYPE[dtype])
    b = Buffer(y=N * ld * size, last=k * D * 4, states=kept * D * 4, workspace=nbytes, flags=4, df=N * ld * size, du=N * ld * size, dh0=k * D * 4)
    b.part("flags", torch.int32, (1,)).zero_()
    stream = torch.cuda.current_stream().cuda_stream
    inputs = (f.data_ptr(), D, u.data_ptr(), D, None, offsets.data_ptr(), int(wide), k, h0.data_ptr())
    p = b.pointer
    rc = lib.chicle_gated_scan(*inputs, N, D, TYPE[dtype], p("y"), ld, p("last"), p("states"), p("workspace"), nbytes, p("flags"), stream)
    assert rc == 0 and int(b.part("flags", torch.int32, (1,))) == (4 if wrong else 0)
    assert b.margins_are_whole(ld, D, size, ("y", "df", "du"))
    assert bool((b.part("df", torch.uint8, (-1,)) == FILL).all())
    y, last, states = (b.part(*x).clone() for x in (("y", dtype, (N, ld)), ("last", F32, (k, D)), ("states", F32, (kept, D))))
    b.part("flags", torch.int32, (1,)).zero_()
    rc = lib.chicle_gated_scan_grad(*inputs, p("states"), dy.data_ptr(), D, dlast.data_ptr(), N, D, TYPE[dtype], p("df"), ld, p("du"), ld, p("dh0"), p("workspace"), nbytes,
                                    p("flags"), stream)
    assert rc == 0 and int(b.part("flags", torch.int32, (1,))) == (4 if wrong else 0)
    assert b.margins_are_whole(ld, D, size, ("y", "df", "du"))
    assert torch.equal(b.part("y", dtype, (N, ld)).view(torch.uint8), y.view(torch.uint8)) and torch.equal(b.part("last", F32, (k, D)).view(torch.uint8), last.view(torch.uint8))
    if not wrong:
        want = ops.gated_scan(f, u, offsets, h0, last=True, states=True)
        assert torch.equal(y[:, :D], want[0]) and torch.equal(last, want[1]) and torch.equal(states, want[2])
        df, du, dh0 = ops.gated_scan_grad(f, u, want[2], dy, offsets, h0, dlast)
        assert torch.equal(b.part("df", dtype, (N, ld))[:, :D], df) and torch.equal(b.part("du", dtype, (N, ld))[:, :D], du)
        assert torch.equal(b.part("dh0", F32, (k, D)), dh0)
