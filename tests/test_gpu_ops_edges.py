"""Edges of the operators on the GPU: tables of one row, destinations too
narrow for their source, derivatives, versions, streams."""
import math

import numpy as np
import pytest

import paper_2511_07035_amd as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [0, 5, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [2049, 513, 8200])
def test_the_gradient_of_a_table_of_one_row_is_written_whole(cols, dtype, tokens):
    """The row stride of a single row means nothing: here it is one element,
    which is also the width of the last block of columns."""
    buf = torch.full((cols + 8,), 9.0, dtype=dtype, device="cuda")
    into = buf[:cols].view(cols, 1).t()
    assert into.shape == (1, cols) and into.stride() == (1, 1)
    ids = torch.full((tokens,), -1, device="cuda")
    g.embedding_grad(torch.ones(tokens, cols, dtype=dtype, device="cuda"), ids, into)
    assert bool((into == 0.0).all()) and bool((buf[cols:] == 9.0).all())
    if tokens:
        ids[0] = 0
        g.embedding_grad(torch.ones(tokens, cols, dtype=dtype, device="cuda"), ids, into)
        assert bool((into == 1.0).all()) and bool((buf[cols:] == 9.0).all())


@pytest.mark.parametrize("rows", [6, 11])
def test_a_gradient_of_another_shape_than_the_table_is_refused(rows):
    table = torch.randn(10, 8, device="cuda").requires_grad_()
    ids = torch.tensor([1, 7, 9, 10], device="cuda")
    with pytest.raises(ValueError):
        g.embedding(table, ids, grad_weight=torch.zeros(rows, 8, device="cuda"))
    for bad in (torch.zeros(10, 7, device="cuda"), torch.zeros(80, device="cuda"), torch.zeros(10, 8),
                torch.zeros(10, 8, dtype=torch.float64, device="cuda")):
        with pytest.raises(ValueError):
            g.embedding(table, ids, grad_weight=bad)
    into = torch.full((10, 8), 5.0, dtype=torch.bfloat16, device="cuda")
    g.embedding(table, ids, grad_weight=into).sum().backward()
    want = torch.zeros(10, 8, device="cuda")
    want[[1, 7, 9]] = 1.0
    assert torch.equal(into.float(), want)


# The smallest fp32 products that round to infinity: half a step above the
# largest finite value, and ties go to even, which here is infinity.
LEAST_INF = {torch.float16: 65520.0, torch.bfloat16: 2.0 ** 128 - 2.0 ** 119}
NARROW = [(torch.float32, torch.float16), (torch.bfloat16, torch.float16), (torch.float32, torch.bfloat16)]


def with_element(n, dtype, at, value):
    t = torch.zeros(n, dtype=dtype, device="cuda")
    t[at] = value
    return t


@pytest.mark.parametrize("again", ["0", "1"])
@pytest.mark.parametrize("src,dst", NARROW)
@pytest.mark.parametrize("n", [1, 20_001, 6_000_001])
def test_found_inf_where_the_destination_is_too_narrow(n, src, dst, again, monkeypatch):
    """Finite gradients whose rounding gives an infinity: the flag is set, at
    the very value from which on the rounding gives one."""
    monkeypatch.setenv("GOCKPT_TEST_GRADS_AGAIN", again)
    least = LEAST_INF[dst]
    below = float(np.nextafter(np.float32(least), np.float32(0)))
    if src == torch.bfloat16:  # the bf16 values around it
        least, below = 65536.0, 65280.0
    out = torch.empty(n, dtype=dst, device="cuda")
    for at in sorted({0, n // 2, n - 1}):
        for value, inf in ((below, 0.0), (-below, 0.0), (least, 1.0), (-least, 1.0)):
            t = with_element(n, src, at, value)
            gl = g.GradList([torch.zeros(3, device="cuda"), t], [None, out])
            r = gl.clip(float("inf"))
            assert float(r.found_inf) == inf and float(r.coef) == 1.0
            assert bool(torch.isinf(out).any()) == bool(inf) and math.isfinite(float(r.norm))
            # scaled into the range: no infinity, no flag
            r = gl.clip(1.0)
            assert float(r.found_inf) == 0.0 and bool(torch.isfinite(out).all())
            # the same gradients in place, or into fp32, round to nothing new
            assert float(g.GradList([t.clone()]).clip(float("inf")).found_inf) == 0.0
            assert float(g.GradList([t], [torch.empty(n, device="cuda")]).clip(float("inf")).found_inf) == 0.0


def test_the_flag_of_a_narrow_destination_among_others():
    """Each destination's own range counts, whatever lies beside it, and a NaN
    or infinity counts as before."""
    def flag(*pairs):
        outs = [None if d is None else torch.empty_like(t, dtype=d) for t, d in pairs]
        return float(g.GradList([t for t, _ in pairs], outs).clip(float("inf")).found_inf)

    big = with_element(5000, torch.float32, 77, 1e30)
    small = with_element(300, torch.float32, 3, 65504.0)
    assert flag((big, torch.bfloat16), (small, torch.float16)) == 0.0
    assert flag((big, torch.float16), (small, torch.bfloat16)) == 1.0
    assert flag((big, None), (small, torch.float16)) == 0.0
    assert flag((big, torch.float32), (small, torch.float16)) == 0.0
    for value in (float("inf"), float("nan")):
        assert flag((big, None), (with_element(9, torch.float32, 2, value), torch.float16)) == 1.0
        assert flag((with_element(9, torch.float16, 2, value), torch.bfloat16)) == 1.0


def test_ranks_put_their_ranges_together():
    """Ranks that hold different parameters add up sumsq and take the larger
    of their ranges: the flag is then that of all of them."""
    a, b = with_element(100, torch.float32, 1, 70000.0), torch.ones(100, device="cuda")
    lists = [g.GradList([t], [torch.empty(100, dtype=torch.float16, device="cuda")]) for t in (a, b)]
    ra, rb = (gl.norm(float("inf")) for gl in lists)
    assert float(ra.found_inf) == 1.0 and float(rb.found_inf) == 0.0
    sumsq, largest = ra.sumsq + rb.sumsq, torch.maximum(ra.largest, rb.largest)
    for most, inf in ((float("inf"), 1.0), (70000.0, 1.0), (65000.0, 0.0)):
        for r in (ra, rb):
            r.sumsq.copy_(sumsq)
            r.largest.copy_(largest)
            r.update(most)
            assert float(r.found_inf) == inf


@pytest.mark.parametrize("n", [40_000, 6_000_000])
def test_a_step_whose_gradients_overflow_in_the_clip_is_skipped(n):
    """fp32 sums over micro-batches clipped into the fp16 gradient of a Session
    that takes the clip's flag: the step is skipped, the scale backs off."""
    result = g.GradResult()
    sess = g.Session(n, ring_bytes=1 << 20, dynamic_scale=True, init_scale=1024.0, found_inf=result.found_inf,
                     grad_norm=False, grad_dtype="fp16")
    try:
        with torch.cuda.stream(sess.compute):
            sess.master.normal_(0.0, 0.02)
            sess.weight.copy_(sess.master)
            sums = torch.full((n,), 0.5, device="cuda")
            gl = g.GradList([sums], [sess.grad], stream=sess.compute)
            before = sess.master.clone()
            sums[n - 5] = 70000.0
            gl.clip(1e9, scale=sess, result=result)
            sess.step(1e-3)
            assert torch.equal(sess.master, before) and float(result.found_inf) == 1.0
            sums[n - 5] = 0.5
            gl.clip(1e9, scale=sess, result=result)
            assert float(result.norm) == float(np.float32(math.sqrt(n) * 0.5 / 512.0))
            sess.step(1e-3)
            assert float(result.found_inf) == 0.0
            assert not torch.equal(sess.master, before) and bool(torch.isfinite(sess.master).all())
    finally:
        sess.close()


@pytest.mark.parametrize("n", [700, 3_000_000, 20_000_001])
def test_no_call_depends_on_another_block(n, monkeypatch):
    """With no polls the block that writes the result computes every partial
    that it does not find: the same bits as with polls, call after call on one
    list whose gradients change."""
    t = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    polled = g.GradList([t])
    monkeypatch.setenv("GOCKPT_TEST_GRADS_AGAIN", "1")
    alone = g.GradList([t])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    for _ in range(9):
        t.normal_(0.0, 1e-3, generator=gen)
        want = float(t.double().square().sum())
        a, b = polled.norm(1e-3).buffer.clone(), alone.norm(1e-3).buffer
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))
        assert abs(float(alone.result.sumsq) - want) <= 34 * 2.0 ** -24 * want


def test_calls_of_one_list_on_several_streams_run_in_order():
    t = torch.zeros(3_000_000, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    gl = g.GradList([t], stream=streams[0])
    results = [g.GradResult() for _ in range(4)]
    torch.cuda.synchronize()
    with torch.cuda.stream(streams[0]):
        torch.cuda._sleep(20_000_000)  # the gradients are written late on the first stream
        t.fill_(2.0)
    for r, s in zip(results, [*streams, streams[0]]):
        gl.norm(result=r, stream=s)
    gl.clip(1.0)  # on the current one
    torch.cuda.synchronize()
    assert [float(r.sumsq) for r in results] == [12e6] * 4
    assert float(gl.result.sumsq) == 12e6 and float(t[-1]) == float(np.float32(2.0) * np.float32(float(gl.result.coef)))
    gl.close()


def test_the_forward_derivative_is_the_lookup_of_the_tangent():
    from torch.autograd import forward_ad
    w, v = torch.randn(12, 5, device="cuda"), torch.randn(12, 5, device="cuda")
    ids = torch.tensor([[1, 5, -1], [11, 12, 5]], device="cuda")
    for need in (False, True):
        with forward_ad.dual_level():
            dual = forward_ad.make_dual(w.clone().requires_grad_(need), v)
            y, dy = forward_ad.unpack_dual(g.embedding(dual, ids, scale=1.5, padding_id=5))
            assert torch.equal(y, g.embedding(w, ids, scale=1.5))
            assert dy is not None and torch.equal(dy, g.embedding(v, ids, scale=1.5))
    with forward_ad.dual_level():  # a tangent of other strides, into another type
        y = g.embedding(forward_ad.make_dual(w, v[:1].expand(12, 5)), ids, out_dtype=torch.bfloat16)
        assert torch.equal(forward_ad.unpack_dual(y).tangent, g.embedding(v[:1].repeat(12, 1), ids,
                                                                          out_dtype=torch.bfloat16))
    with forward_ad.dual_level():  # no tangent: none comes out
        assert forward_ad.unpack_dual(g.embedding(w, ids)).tangent is None
        with pytest.raises(ValueError):
            g.embedding(forward_ad.make_dual(w, v), ids, out=torch.empty(2, 3, 5, device="cuda"))


def test_an_out_that_requires_a_gradient_is_refused():
    w, ids = torch.randn(12, 5, device="cuda"), torch.tensor([1, 5], device="cuda")
    out = torch.zeros(2, 5, device="cuda", requires_grad=True)
    with pytest.raises(ValueError):
        g.embedding(w, ids, out=out)
    with torch.no_grad():
        assert torch.equal(g.embedding(w, ids, out=out), w[ids])


def test_a_buffer_that_autograd_saved_cannot_change_unseen():
    """What a call writes in place counts as a change of the tensor, of its
    base and of its views."""
    w, ids = torch.randn(12, 5, device="cuda"), torch.tensor([1, 5], device="cuda")
    base = torch.ones(200, device="cuda")
    calls = [lambda t: g.embedding(w, ids, out=t.view(2, 5)),
             lambda t: g.embedding_grad(torch.ones(2, 5, device="cuda"), ids % 2, t.view(2, 5)),
             lambda t: g.GradList([t]).clip(0.1),
             lambda t: g.GradList([torch.ones(10, device="cuda")], [t]).clip(0.1),
             lambda t: g.GradList([t]).scale(g.GradList([torch.ones(9, device="cuda")]).norm(0.1))]
    for call in calls:
        for buf in (torch.ones(10, device="cuda"), base[3:13]):
            x = torch.ones(10, device="cuda", requires_grad=True)
            loss = (x * buf).sum()
            call(buf)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                loss.backward()
    with torch.inference_mode():  # tensors without a version
        t = torch.ones(10, device="cuda")
        for call in calls:
            call(t)
    # a norm reads its tensors
    x, t = torch.ones(10, device="cuda", requires_grad=True), torch.ones(10, device="cuda")
    loss = (x * t).sum()
    gl = g.GradList([t], [torch.empty(10, device="cuda")])
    gl.norm(0.1)
    gl.clip(0.1)
    loss.backward()
    assert torch.equal(x.grad, t)


def test_a_call_beside_a_session_waits_for_its_steps_scale():
    flag = torch.ones(1, device="cuda")
    sess = g.Session(5000, ring_bytes=1 << 20, dynamic_scale=True, init_scale=1024.0, found_inf=flag, grad_norm=False)
    try:
        t, other = torch.full((100,), 512.0, device="cuda"), torch.cuda.Stream()
        torch.cuda.synchronize()
        gl = g.GradList([t])
        torch.cuda.synchronize()
        with torch.cuda.stream(sess.compute):
            torch.cuda._sleep(20_000_000)  # the step that halves the scale runs late
        sess.step(1e-3)
        beside = gl.norm(scale=sess, result=g.GradResult())
        updated = g.GradResult()
        updated.sumsq.fill_(100 * 512.0 ** 2)
        torch.cuda.synchronize()
        with torch.cuda.stream(sess.compute):
            torch.cuda._sleep(20_000_000)
        sess.step(1e-3)
        updated.update(scale=sess, stream=other)
        torch.cuda.synchronize()
        assert float(beside.norm) == 10.0 and float(updated.norm) == 20.0
    finally:
        sess.close()


def test_a_table_without_columns():
    w, ids = torch.zeros(10, 0, device="cuda"), torch.tensor([[1, 5, 11]], device="cuda")
    assert g.embedding(w, ids).shape == (1, 3, 0)
    assert g.embedding(w, ids, out=torch.zeros(1, 3, 0, device="cuda")).shape == (1, 3, 0)
    into = torch.zeros(10, 0, device="cuda")
    assert g.embedding_grad(torch.zeros(1, 3, 0, device="cuda"), ids, into) is into
    w.requires_grad_()
    g.embedding(w, ids).sum().backward()
    assert w.grad.shape == (10, 0)


def test_a_list_that_ends_while_a_graph_records():
    """Closing a list whose calls ran on another stream waits for nothing that
    a recording forbids."""
    t, x, other = torch.ones(5000, device="cuda"), torch.zeros(4, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    lists = [g.GradList([t]) for _ in range(2)]
    for gl in lists:
        gl.norm(stream=other)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1.0)
        lists.pop().close()
        lists.clear()
        x.add_(1.0)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert float(x[0]) == 2.0 * (k + 1)
