"""How the training operators are called: from several threads, on several streams, into graphs, beside automatic differentiation."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ops():
    import paper_1909_04885_amd as chicle
    return chicle.TrainOps("cuda:0")


def test_the_first_calls_come_from_several_threads(ops):
    """All of them report to one word, which lives as long as the kernels that look at it."""
    import paper_1909_04885_amd as chicle
    word = ops._flags()
    table, ids = torch.randn(10, 24, device="cuda"), torch.arange(8, device="cuda", dtype=torch.int32)
    past = torch.full((3,), 10, device="cuda", dtype=torch.int32)
    seen, begin = [], threading.Barrier(8)

    def work(k):
        begin.wait()
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                ops.embed(table, ids)
            if k == 5:
                ops.embed(table, past)
            seen.append(ops._flags())
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(k,)) for k in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert set(seen) == {word} and len(seen) == 8
    with pytest.raises(chicle.ChicleError, match="token"):
        ops.sync()
    ops.sync()


def test_a_report_is_taken_by_one_sync_and_none_is_lost(ops):
    """Syncs of several threads, each behind its own report: every report is raised once at least, and none is left."""
    import paper_1909_04885_amd as chicle
    table, past = torch.randn(10, 24, device="cuda"), torch.full((3,), 10, device="cuda", dtype=torch.int32)
    x, w, label = torch.randn(3, 24, device="cuda"), torch.randn(5, 24, device="cuda"), torch.full((3,), 5, device="cuda", dtype=torch.int32)
    raised = []

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(50):
                ops.embed(table, past) if k % 2 else ops.softmax_loss(x, w, label)
                try:
                    ops.sync()
                except chicle.ChicleError as e:
                    raised.append(str(e))

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    ops.sync()
    assert any("token" in s for s in raised) and any("label" in s for s in raised)


def test_the_first_call_may_be_captured(ops):
    table, ids = torch.randn(50, 24, device="cuda"), torch.arange(20, device="cuda", dtype=torch.int32)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.embed(table, ids, 2.0)
    for k in range(3):
        ids.copy_(torch.randint(0, 50, (20,), device="cuda", dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, table[ids.long()] * 2.0), k
    ids[4] = 50
    graph.replay()
    import paper_1909_04885_amd as chicle
    with pytest.raises(chicle.ChicleError, match="token"):
        ops.sync()


def test_what_requires_a_gradient_is_refused_while_gradients_are_recorded(ops):
    import paper_1909_04885_amd as chicle
    x, w, v, ids = torch.randn(4, 8, device="cuda"), torch.randn(10, 8, device="cuda"), torch.ones(8, device="cuda"), torch.arange(4, device="cuda")
    ones = torch.ones(4, device="cuda")

    def calls(x, w, v, ones):
        yield lambda: ops.softmax_loss(x, w, ids)
        yield lambda: ops.softmax_loss_grad(x, w, ids, ones)
        yield lambda: ops.embed(w, ids)
        yield lambda: ops.embed_grad(ids, x, 10)
        yield lambda: ops.embed_grad(ids, x.detach(), 10, into=w)
        yield lambda: ops.layer_norm(x, v, v.detach())
        yield lambda: ops.layer_norm_grad(x, x.detach(), v.detach(), ones.detach(), ones.detach())

    asked = [t.clone().requires_grad_() for t in (x, w, v, ones)]
    for k, call in enumerate(calls(*asked)):
        with pytest.raises(chicle.ChicleError, match="requires a gradient"):
            call()
            pytest.fail("call %d was not refused" % k)
    with torch.no_grad():
        for call in calls(*asked):
            call()
    for call in calls(x, w, v, ones):
        call()
    with torch.inference_mode():
        ops.clip_grads([torch.ones(5, device="cuda")], 1.0)


def test_what_is_written_in_place_has_a_new_version(ops):
    a = torch.randn(6, 8, device="cuda", requires_grad=True)
    for write in (lambda t: ops.clip_grads([t], 1.0), lambda t: ops.clip_grads([torch.ones_like(t)], 1.0, [t]),
                  lambda t: ops.embed_grad(torch.arange(6, device="cuda"), torch.ones_like(t), 6, into=t)):
        saved = torch.randn(6, 8, device="cuda")
        product = (a * saved).sum()
        write(saved)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            product.backward()
    saved = torch.randn(6, 8, device="cuda")
    product = (a * saved).sum()
    ops.grad_norm([saved])
    ops.clip_grads([saved], 1.0, [torch.empty_like(saved)])
    product.backward()


def test_memory_that_would_be_written_twice_is_refused(ops):
    """Two workgroups would scale it beside each other, each what the other may have scaled."""
    import paper_1909_04885_amd as chicle
    a, b, empty = torch.ones(50000, device="cuda"), torch.ones(7, device="cuda"), torch.empty(0, device="cuda")
    for call in (lambda: ops.clip_grads([a, b, a], 1.0), lambda: ops.clip_grads([a, a], 1.0, [b.new_empty(50000)] * 2),
                 lambda: ops.clip_grads([b, a[100:], a[:101]], 1.0)):
        with pytest.raises(chicle.ChicleError, match="twice"):
            call()
    assert a.eq(1).all()
    assert abs(float(ops.grad_norm([a, a])) - 100000 ** 0.5) < 1e-3      # (read twice it may be)
    ops.clip_grads([a, a], 1.0, [torch.empty_like(a), torch.empty_like(a)])
    ops.clip_grads([a[100:], a[:100]], 1e9)
    ops.clip_grads([empty, b, empty, empty[:0]], 1.0)


def test_layer_norm_of_rows_whose_columns_fill_more_than_a_launch(ops):
    """2^25 columns and more: the sums over rows of the gradients by weight and bias have 2 d columns, 16 to a workgroup of 1024 threads."""
    n, d = 2, (1 << 25) + 21
    print("\ncase layer_norm_grad", n, d, flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x, dy = (torch.randn(n, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    gamma = (torch.rand(d, generator=g, device="cuda") + 0.5).to(torch.bfloat16)
    _, mean, rstd = ops.layer_norm(x, gamma, gamma)
    dx, dgamma, dbeta = ops.layer_norm_grad(dy, x, gamma, mean, rstd)
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    # two terms of each sum, and the rounding of the result
    for got, terms in ((dgamma, dy.double() * h), (dbeta, dy.double())):
        want = terms.sum(0)
        assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * terms.abs().sum(0)).all())


def test_gradient_of_a_table_whose_rows_fill_more_than_a_launch(ops):
    """2^24 rows of 8200 bytes: zeros for a row or two to a workgroup."""
    n_rows, d = (1 << 24) + 3, 4100
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("138 GB are not free")
    print("\ncase embed_grad", n_rows, d, flush=True)
    before = torch.ones(n_rows, d, dtype=torch.bfloat16, device="cuda")
    at = before.data_ptr()
    del before                                           # (the result's memory, which holds ones)
    ids = torch.tensor([n_rows - 1, 5, -1, 5, 1 << 23], device="cuda")
    dout = torch.randn(5, d, device="cuda").to(torch.bfloat16)
    got = ops.embed_grad(ids, dout, n_rows)
    assert got.data_ptr() == at
    assert torch.equal(got[n_rows - 1], dout[0]) and torch.equal(got[1 << 23], dout[4])
    assert torch.equal(got[5], (dout[1].float() + dout[3].float()).to(torch.bfloat16))
    got[ids[[0, 1, 4]]] = 0
    step = 1 << 20
    for a in range(0, n_rows, step):
        assert not got[a:a + step].any(), a
    del got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [32736, 32737, 40001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_gradient_of_a_table_about_where_pieces_get_longer(ops, dtype, n):
    import train_reference as ref
    d, n_rows = 1100, 700
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    ids = torch.randint(-1, n_rows, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[5000:9000] = 7                                   # a run over many pieces
    dout = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    want, off = ref.embed_grad(ids, dout, n_rows, 0.7)
    got = ops.embed_grad(ids, dout, n_rows, 0.7)
    ref.within(got, want, off)
    assert torch.equal(got, ops.embed_grad(ids, dout, n_rows, 0.7))
