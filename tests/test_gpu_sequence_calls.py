"""How the operators of layers over sequences are called: into graphs, on several streams, beside automatic differentiation, on a lot of memory."""
import pytest
import torch

import sequence_reference as ref
from train_reference import TINY, U, within

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAN, INF = float("nan"), float("inf")


@pytest.fixture()
def ops():
    import paper_1909_04885_amd as chicle
    return chicle.TrainOps("cuda:0")


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def layer(ops, x, res, gamma, f, offsets, dy, keep8):
    """Forward and backward of one layer, as local SGD has it."""
    y, r, rstd, kept = ops.rms_norm(x, gamma, res, y8=keep8, keep8=keep8)
    h, last, states = ops.gated_scan(f, y, offsets, last=True, states=True)
    df, du, _ = ops.gated_scan_grad(f, y, states, dy, offsets)
    dx, dgamma = ops.rms_norm_grad(du, kept if keep8 else r, gamma, rstd, dy)
    return h, last, states, df, du, dx, dgamma


@pytest.mark.parametrize("keep8", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_layer_in_a_graph(ops, dtype, keep8):
    """Replayed several times with other inputs, and eager work between: every replay gives what eager calls give, bit for bit."""
    g = gen(1)
    n, d = 1300, 200
    x, res, f, dy = (torch.randn(n, d, generator=g, device="cuda").to(dtype) for _ in range(4))
    gamma = torch.rand(d, generator=g, device="cuda").to(dtype)
    offsets = torch.tensor([0, 3, 3, 700, 701, 1290], dtype=torch.int32, device="cuda")
    layer(ops, x, res, gamma, f, offsets, dy, keep8)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):                                   # two graphs of one pool
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=graphs[0][0].pool() if graphs else None):
            out = layer(ops, x, res, gamma, f, offsets, dy, keep8)
        graphs.append((graph, out))
    for k in range(6):
        for t in (x, res, f, dy):
            t.copy_(torch.randn(n, d, generator=g, device="cuda"))
        offsets[1:3] = 3 + 40 * k
        want = [t.clone() for t in layer(ops, x, res, gamma, f, offsets, dy, keep8)]
        graph, out = graphs[k % 2]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want)), k
    ops.sync()


def test_steps_in_a_graph_go_on(ops):
    g = gen(2)
    f, u, state = torch.randn(9, 70, generator=g, device="cuda"), torch.randn(9, 70, generator=g, device="cuda"), torch.zeros(9, 70, device="cuda")
    ops.gated_step(f, u, state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ops.gated_step(f, u, state)
    want = state.clone()
    for k in range(5):
        u.copy_(torch.randn(9, 70, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        w = ops.gated_step(f, u, want)
        assert torch.equal(y, w) and torch.equal(state, want), k


def test_scans_on_several_streams_at_once(ops):
    """Scans whose tiles wait for one another, beside each other on the chip: each gives what it gives alone, every time."""
    g = gen(3)
    cases = []
    for k, (n, d) in enumerate([(9000, 512), (20000, 300), (5000, 1100), (70000, 64)]):
        f, u = (torch.randn(n, d, generator=g, device="cuda").to((F32, BF16)[k % 2]) for _ in range(2))
        y, _, states = ops.gated_scan(f, u, states=True)
        cases.append((f, u, y, states, ops.gated_scan_grad(f, u, states, y)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = []
    for _ in range(8):
        for s, (f, u, y, states, _) in zip(streams, cases):
            with torch.cuda.stream(s):
                got.append((ops.gated_scan(f, u)[0], ops.gated_scan_grad(f, u, states, y)))
    torch.cuda.synchronize()
    for k, (y, grads) in enumerate(got):
        _, _, want, _, want_grads = cases[k % 4]
        assert torch.equal(y, want) and torch.equal(grads[0], want_grads[0]) and torch.equal(grads[1], want_grads[1]), k


def test_what_requires_a_gradient_is_refused_while_gradients_are_recorded(ops):
    import paper_1909_04885_amd as chicle
    x, v, ones = torch.randn(40, 8, device="cuda"), torch.ones(8, device="cuda"), torch.ones(40, device="cuda")
    state, states = torch.zeros(1, 8, device="cuda"), torch.zeros(2, 8, device="cuda")

    def calls(x, v, ones, state, states):
        yield lambda: ops.pack8(x)
        yield lambda: ops.rms_norm(x, v.detach())
        yield lambda: ops.rms_norm(x.detach(), v)
        yield lambda: ops.rms_norm(x.detach(), v.detach(), x)
        yield lambda: ops.rms_norm_grad(x, x.detach(), v.detach(), ones.detach())
        yield lambda: ops.rms_norm_grad(x.detach(), x.detach(), v.detach(), ones)
        yield lambda: ops.rms_norm_grad(x.detach(), x.detach(), v.detach(), ones.detach(), x)
        yield lambda: ops.gated_scan(x, x.detach())
        yield lambda: ops.gated_scan(x.detach(), x.detach(), None, state)
        yield lambda: ops.gated_scan_grad(x.detach(), x.detach(), states, x.detach())
        yield lambda: ops.gated_scan_grad(x.detach(), x.detach(), states.detach(), x)
        yield lambda: ops.gated_scan_grad(x.detach(), x.detach(), states.detach(), x.detach(), None, None, state)
        yield lambda: ops.gated_step(x[:1].detach(), x[:1].detach(), state)

    asked = [t.clone().requires_grad_() for t in (x, v, ones, state, states)]
    for k, call in enumerate(calls(*asked)):
        with pytest.raises(chicle.ChicleError, match="requires a gradient"):
            call()
            pytest.fail("call %d was not refused" % k)
    with torch.no_grad():
        for call in calls(*asked):
            call()
    with torch.inference_mode():
        ops.gated_step(x[:1].clone(), x[:1].clone(), state.clone())


def test_a_state_that_is_written_has_a_new_version(ops):
    a, x = torch.randn(6, 8, device="cuda", requires_grad=True), torch.randn(6, 8, device="cuda")
    state = torch.randn(6, 8, device="cuda")
    product = (a * state).sum()
    ops.gated_step(x, x, state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.backward()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_states_that_lie_between_the_rows_of_other_tensors(ops, dtype):
    """One buffer has the rows of f, u and the states beside each other, the states first or last; what is between stays as it was."""
    g, n, d = gen(9), 5, 24
    f, u, state = torch.randn(n, d, generator=g, device="cuda").to(dtype), torch.randn(n, d, generator=g, device="cuda").to(dtype), torch.randn(n, d, generator=g, device="cuda")
    want_state = state.clone()
    want = ops.gated_step(f, u, want_state)
    narrow = d * f.element_size() // 4                   # floats that a row of f takes
    for first in (0, 2 * narrow):
        buffer = torch.zeros(n, 2 * narrow + d, device="cuda")
        at = d if first == 0 else 0
        s = buffer[:, first:first + d]
        rows = [buffer[:, at + k * narrow:at + (k + 1) * narrow].view(dtype) for k in range(2)]
        s.copy_(state), rows[0].copy_(f), rows[1].copy_(u)
        assert torch.equal(ops.gated_step(*rows, s), want) and torch.equal(s, want_state) and torch.equal(rows[0], f) and torch.equal(rows[1], u)
    wide = torch.zeros(n, d, device="cuda")
    for bad in ((wide, f.float()), (f.float(), wide)):
        with pytest.raises(Exception, match="overlap"):
            ops.gated_step(*bad, wide)
    ops.sync()


def test_refusals(ops):
    import paper_1909_04885_amd as chicle
    x, v, ones = torch.randn(40, 64, device="cuda"), torch.ones(64, device="cuda"), torch.ones(40, device="cuda")
    half, p, states = x.to(BF16), ops.pack8(x), torch.zeros(2, 64, device="cuda")
    off = torch.tensor([0, 40], device="cuda")
    bad = [
        lambda: ops.pack8(x.t()), lambda: ops.pack8(x.cpu()), lambda: ops.pack8(x.double()), lambda: ops.pack8(x[0]),
        lambda: ops.unpack8(p, torch.float64), lambda: ops.unpack8(chicle.Packed8(p.values, p.scales, 65), F32), lambda: ops.unpack8(chicle.Packed8(p.values[:, :32], p.scales[:, :1], 32), F32),
        lambda: ops.unpack8(chicle.Packed8(p.values, p.scales[:39], 64), F32), lambda: ops.unpack8(chicle.Packed8(p.values.cpu(), p.scales.cpu(), 64), F32),
        lambda: ops.unpack8(chicle.Packed8(p.values.view(torch.uint8), p.scales, 64), F32),
        lambda: ops.rms_norm(x, v[:63]), lambda: ops.rms_norm(x, v.to(BF16)), lambda: ops.rms_norm(x, v, half), lambda: ops.rms_norm(x, v, x[:39]),
        lambda: ops.rms_norm(x, v, eps=-1.0), lambda: ops.rms_norm_grad(x, x[:39], v, ones), lambda: ops.rms_norm_grad(x, half, v, ones),
        lambda: ops.rms_norm_grad(x, chicle.Packed8(p.values[:39], p.scales[:39], 64), v, ones), lambda: ops.rms_norm_grad(x, x, v, ones[:39]),
        lambda: ops.rms_norm_grad(x, x, v, ones, x[:39]),
        lambda: ops.gated_scan(x, half), lambda: ops.gated_scan(x, x[:39]), lambda: ops.gated_scan(x, x, off.float()), lambda: ops.gated_scan(x, x, off[:0]),
        lambda: ops.gated_scan(x, x, off, states), lambda: ops.gated_scan(x, x, off, states[:1].to(BF16)), lambda: ops.gated_scan(x, x, torch.stack([off, off], 1)[:, 0]),
        lambda: ops.gated_scan(x, chicle.Packed8(p.values[:39], p.scales[:39], 64)),
        lambda: ops.gated_scan_grad(x, x, states[:1], x), lambda: ops.gated_scan_grad(x, x, states, x[:39]), lambda: ops.gated_scan_grad(x, x, states, half),
        lambda: ops.gated_scan_grad(x, x, states, x, off, None, states),
        lambda: ops.gated_step(x, x, half), lambda: ops.gated_step(x, x, x[:39]), lambda: ops.gated_step(x, x[:39], x.clone()),
        lambda: ops.gated_step(x, x, torch.zeros(1, 64, device="cuda").expand(40, 64)), lambda: ops.gated_step(x, p, x.clone())]
    for k, call in enumerate(bad):
        with pytest.raises(chicle.ChicleError):
            call()
            pytest.fail("call %d was not refused" % k)
    ops.sync()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_nothing_of_a_sequence_reaches_another(ops, dtype):
    """Infinities and NaN in the rows, gates, states and gradients of some sequences: the others get the same bits as without."""
    g = gen(5)
    n, d = 700, 70
    at = [0, 1, 40, 40, 128, 129, 300, 512, 640, 641, 700]
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    f, u, dy = (torch.randn(n, d, generator=g, device="cuda").to(dtype) for _ in range(3))
    h0, dlast = (torch.randn(len(at) - 1, d, generator=g, device="cuda") for _ in range(2))
    for a, b in ((None, None), (h0, None), (None, dlast), (h0, dlast)):
        y, last, states = ops.gated_scan(f, u, offsets, a, last=True, states=True)
        grads = ops.gated_scan_grad(f, u, states, dy, offsets, a, b)
        again = ops.gated_scan_grad(f, u, states, dy, offsets, a, b)
        assert all(p is q or torch.equal(p, q) for p, q in zip(grads, again)) and torch.equal(y, ops.gated_scan(f, u, offsets, a)[0])
        bad = [1, 5, 7]
        df, du, dd, da, db = f.clone(), u.clone(), dy.clone(), None if a is None else a.clone(), None if b is None else b.clone()
        for k, j in enumerate(bad):
            lo, hi = at[j], at[j + 1]
            du[lo + (hi - lo) // 2], dd[hi - 1, ::2], df[lo, 1::3] = NAN if k else INF, NAN, NAN
            for t in (da, db):
                if t is not None:
                    t[j] = (INF, NAN, -INF)[k]
        rows = torch.ones(n, dtype=torch.bool, device="cuda")
        for j in bad:
            rows[at[j]:at[j + 1]] = False
        others = torch.tensor([j for j in range(len(at) - 1) if j not in bad], device="cuda")
        y2, last2, states2 = ops.gated_scan(df, du, offsets, da, last=True, states=True)
        assert torch.equal(y2[rows], y[rows]) and torch.equal(last2[others], last[others])
        grads2 = ops.gated_scan_grad(df, du, states2, dd, offsets, da, db)
        assert torch.equal(grads2[0][rows], grads[0][rows]) and torch.equal(grads2[1][rows], grads[1][rows])
        if a is not None:
            assert torch.equal(grads2[2][others], grads[2][others])
    ops.sync()


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("share", [0.0, -9.0])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_what_is_no_number_goes_on_until_a_gate_is_closed(ops, dtype, share, bad):
    """Also where the product of the shares between is too small for a number: a half or 1.2e-4 a row."""
    n, d, first, shut = 900, 70, 3, 700
    f, u = torch.full((n, d), share, dtype=dtype, device="cuda"), torch.ones(n, d, dtype=dtype, device="cuda")
    u[first, ::2] = bad
    f[shut, ::4] = -INF
    offsets = torch.tensor([0, 850, n], device="cuda")
    y, last, states = ops.gated_scan(f, u, offsets, last=True, states=True)
    assert not y[first:shut, ::2].isfinite().any() and not y[shut:850, 2::4].isfinite().any() and not last[0, 2::4].isfinite().any()
    assert y[:first].isfinite().all() and y[:, 1::2].isfinite().all() and y[shut:, ::4].isfinite().all() and y[850:].isfinite().all()
    dy = torch.ones(n, d, dtype=dtype, device="cuda")
    u[first, ::2] = 1
    dy[845, ::2] = bad
    _, _, states = ops.gated_scan(f, u, offsets, states=True)
    df, du, dh0 = ops.gated_scan_grad(f, u, states, dy, offsets, h0=torch.zeros(2, d, device="cuda"))
    assert not du[shut:846, ::2].isfinite().any() and not du[:shut, 2::4].isfinite().any() and not dh0[0, 2::4].isfinite().any()
    assert du[846:].isfinite().all() and du[:, 1::2].isfinite().all() and du[:shut, ::4].isfinite().all() and dh0[1].isfinite().all()


def test_one_state_and_no_gradient_of_the_last_and_the_other_way_round(ops):
    g = gen(6)
    n, d, at = 300, 33, [0, 100, 100, 290]
    offsets = torch.tensor(at, device="cuda")
    f, u, dy = (torch.randn(n, d, generator=g, device="cuda") for _ in range(3))
    h0, dlast = (torch.randn(3, d, generator=g, device="cuda") for _ in range(2))
    for a, b in ((h0, None), (None, dlast)):
        _, _, states = ops.gated_scan(f, u, offsets, a, states=True)
        got = ops.gated_scan_grad(f, u, states, dy, offsets, a, b)
        w = ref.scan_grad(f.cpu(), u.cpu(), at, None if a is None else a.cpu(), dy.cpu(), None if b is None else b.cpu())
        for name, x in zip(("df", "du", "dh0"), got):
            if x is not None:
                within(x.cpu(), w[name], w["off_" + name], name)


def test_sequences_without_rows_by_the_thousand(ops):
    """Far more sequences than rows: nearly all are empty, many at the same row."""
    g = gen(7)
    n, d, k = 300, 40, 50000
    cuts = torch.randint(0, n + 1, (k - 1,), generator=g, device="cuda").sort().values
    cuts[1000:30000] = cuts[1000]
    cuts = cuts.sort().values
    offsets = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), n)]).to(torch.int32)
    f, u, dy = (torch.randn(n, d, generator=g, device="cuda") for _ in range(3))
    h0, dlast = (torch.randn(k, d, generator=g, device="cuda") for _ in range(2))
    y, last, states = ops.gated_scan(f, u, offsets, h0, last=True, states=True)
    df, du, dh0 = ops.gated_scan_grad(f, u, states, dy, offsets, h0, dlast)
    some = (offsets[1:] > offsets[:-1])
    assert torch.equal(last[~some], h0[~some]) and torch.equal(dh0[~some], dlast[~some])
    at = [0] + offsets[1:][some].tolist()
    which = some.nonzero()[:, 0]
    short = torch.tensor(at, dtype=torch.int32, device="cuda")
    y2, last2, states2 = ops.gated_scan(f, u, short, h0[which], last=True, states=True)
    assert torch.equal(y, y2) and torch.equal(last[some], last2) and torch.equal(states, states2)
    got = ops.gated_scan_grad(f, u, states, dy, short, h0[which], dlast[which])
    assert torch.equal(df, got[0]) and torch.equal(du, got[1]) and torch.equal(dh0[some], got[2])
    ops.sync()


@pytest.mark.parametrize("n, d", [(3, 200000), (200, 40000), (1000000, 1), (131073, 7)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scans_of_wide_and_of_long_rows(ops, dtype, n, d):
    """Against itself in two pieces, which meet the formula elsewhere: the second goes on from the first one's states."""
    print("\ncase scan", dtype, n, d, flush=True)
    g = gen(n)
    f, u, dy = (torch.randn(n, d, generator=g, device="cuda").to(dtype) for _ in range(3))
    cut = n // 3 * 2
    y, last, states = ops.gated_scan(f, u, last=True, states=True)
    y1, mid, states1 = ops.gated_scan(f[:cut], u[:cut], last=True, states=True)
    y2, last2, states2 = ops.gated_scan(f[cut:], u[cut:], None, mid, last=True, states=True)
    near = lambda p, q, t: bool(((p.float() - q.float()).abs() <= 2 * U[t] * q.float().abs() + 1e-5).all())  # noqa: E731  (states of about one, 1e-5: 160 roundings)
    assert near(torch.cat([y1, y2]), y, dtype) and near(last2, last, F32)
    df, du, _ = ops.gated_scan_grad(f, u, states, dy)
    b2 = ops.gated_scan_grad(f[cut:], u[cut:], states2, dy[cut:], None, mid)
    b1 = ops.gated_scan_grad(f[:cut], u[:cut], states1, dy[:cut], None, None, b2[2])
    assert near(torch.cat([b1[0], b2[0]]), df, dtype) and near(torch.cat([b1[1], b2[1]]), du, dtype)


def test_offsets_that_pass_32_bits_in_memory(ops):
    """1.2 million rows of 2048 in 16 bits: more than 2^31 values of each."""
    n, d = 1200000, 2048
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("60 GB are not free")
    print("\ncase", n, d, flush=True)
    g = gen(8)
    f = torch.empty(n, d, dtype=BF16, device="cuda").normal_(1.0, 1.0, generator=g)
    u = torch.empty(n, d, dtype=BF16, device="cuda").normal_(generator=g)
    gamma = torch.ones(d, dtype=BF16, device="cuda")
    tail = slice(n - 500, n)
    offsets = torch.tensor([0, 77, n - 500, n], dtype=torch.int32, device="cuda")
    y, _, states = ops.gated_scan(f, u, offsets, states=True)
    want, _, tail_states = ops.gated_scan(f[tail], u[tail], states=True)
    assert bool(((y[tail].float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 1e-5).all())
    df, du, _ = ops.gated_scan_grad(f, u, states, y, offsets)
    wf, wu, _ = ops.gated_scan_grad(f[tail], u[tail], tail_states, y[tail])
    assert bool(((df[tail].float() - wf.float()).abs() <= 2.0 ** -7 * wf.float().abs() + 1e-4).all())
    assert bool(((du[tail].float() - wu.float()).abs() <= 2.0 ** -7 * wu.float().abs() + 1e-4).all())
    del df, du, states
    p = ops.pack8(u)
    q = ops.pack8(u[tail])
    assert torch.equal(p.values[tail], q.values) and torch.equal(p.scales[tail], q.scales) and torch.equal(ops.unpack8(p, BF16)[tail], ops.unpack8(q, BF16))
    yn, r, rstd, kept = ops.rms_norm(u, gamma, f, y8=True, keep8=True)
    yt, rt, rstdt, keptt = ops.rms_norm(u[tail], gamma, f[tail], y8=True, keep8=True)
    assert torch.equal(r[tail], rt) and torch.equal(yn.values[tail], yt.values) and torch.equal(kept.values[tail], keptt.values)
    dx, _ = ops.rms_norm_grad(y, kept, gamma, rstd, f)
    assert torch.equal(dx[tail], ops.rms_norm_grad(y[tail], keptt, gamma, rstdt, f[tail])[0])
    ops.sync()
    torch.cuda.empty_cache()


def test_norm_of_rows_that_fill_more_than_a_launch(ops):
    """2^25 columns and more, and 2^24 rows."""
    n, d = 2, (1 << 25) + 21
    print("\ncase rms_norm", n, d, flush=True)
    g = gen(9)
    x, dy = (torch.empty(n, d, dtype=BF16, device="cuda").normal_(generator=g) for _ in range(2))
    gamma = (torch.rand(d, generator=g, device="cuda") + 0.5).to(BF16)
    _, _, rstd, kept = ops.rms_norm(x, gamma, keep8=True)
    _, dgamma = ops.rms_norm_grad(dy, x, gamma, rstd)
    terms = dy.double() * x.double() * rstd.double()[:, None]
    want = terms.sum(0)
    # two terms of each sum, and the rounding of the result
    assert bool(((dgamma.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * terms.abs().sum(0)).all())
    del terms, want
    x = torch.empty((1 << 24) + 5, 3, dtype=F32, device="cuda").normal_(generator=g)
    gamma = torch.ones(3, device="cuda")
    y, _, rstd, kept = ops.rms_norm(x, gamma, keep8=True)
    last = ops.rms_norm(x[-7:], gamma, keep8=True)
    assert torch.equal(y[-7:], last[0]) and torch.equal(kept.values[-7:], last[3].values)
    dx, _ = ops.rms_norm_grad(y, kept, gamma, rstd)
    assert torch.equal(dx[-7:], ops.rms_norm_grad(last[0], last[3], gamma, last[2])[0])
