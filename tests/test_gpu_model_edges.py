"""Edges of the model's operators on the GPU.  Tolerances as in test_gpu_model,
whose helpers these tests take."""
import copy
import ctypes
import math
import pickle

import pytest

import paper_2511_07035_amd as g
from paper_2511_07035_amd import model, ops

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_model import (DT, H, U, act64, assert_close, head64, head_inputs, kept64,  # noqa: E402
                            padded, product_error, randn, rounded)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_a_copy_of_8_bits_outlives_the_first(dtype):
    x, other = randn((70, 100), DT[dtype], 1), randn((70, 100), DT[dtype], 2)
    for copied in (copy.deepcopy, lambda a: pickle.loads(pickle.dumps(a))):
        a = g.act8_pack(x)
        b = copied(a)
        g.act8_pack(other, out=a)  # the first one's memory is used for something else
        assert torch.equal(b.unpack().double(), kept64(x))
        g.act8_pack(x, out=a)
        g.act8_pack(other, out=b)  # and writing the copy leaves the first alone
        assert torch.equal(a.unpack().double(), kept64(x)) and torch.equal(b.unpack().double(), kept64(other))
    if dtype != "fp32":
        dy, into = randn((70, 24), DT[dtype], 3), torch.zeros(24, 100, device="cuda")
        g.linear8_grad_weight(dy, b, into)
        K = kept64(other)
        want = dy.double().t() @ K
        assert_close(into, want, product_error(dy.double().t(), K, want, torch.float32))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("tokens,vocab", [(2, 300), (20, 300), (129, 40_000), (256, 300), (256, 40_000), (257, 300)])
def test_head_masked_tokens_beside_infinities(tokens, vocab, value, dtype):
    """A table row with an infinity has the logit -inf, and so no part in the loss
    of the tokens that count; the masked ones add nothing to its gradient either,
    whatever their rows hold."""
    hidden, table, targets = head_inputs(tokens, vocab, 64, dtype)
    hidden[:, 3] = -2.0
    targets[targets == 250] = 7
    table[250, 3] = float("inf")
    hidden[::2] = value
    targets[::2] = -1
    x, w = hidden.detach().requires_grad_(), table.detach().requires_grad_()
    loss = g.linear_cross_entropy(x, w, targets, reduction="none")
    up = randn((tokens,), torch.float32, 5)
    up[::2] = value
    loss.backward(up)
    X, W, y = hidden[1::2].double(), table.double(), targets[1::2]
    n = y.numel()
    logits = X @ W.t()
    assert bool((logits[:, 250] == -math.inf).all())
    W[250] = 0.0
    d = 2 * U * (64 + 2) * (X.abs() @ W.abs().t()) + 2 * U * (X @ W.t()).abs()
    lse = torch.logsumexp(logits, 1)
    e = d.amax(1) + (300 + 8) * U + 4 * U * (lse.abs() + (X @ W.t()).abs().amax(1))
    own = logits.gather(1, y[:, None])[:, 0]
    assert_close(loss.detach()[1::2], lse - own, 2 * e, "loss")
    assert bool((loss.detach()[::2] == 0).all()) and bool((x.grad[::2] == 0).all())
    p = torch.exp(logits - lse[:, None])
    z = p.clone()
    z[torch.arange(n, device="cuda"), y] -= 1.0
    gt = up[1::2].double()
    z *= gt[:, None]
    z_err = gt.abs()[:, None] * p * (d + e[:, None] + 2.0 ** -22) + 4 * U * z.abs() + H[DT[dtype]][0] * z.abs() + \
        2.0 ** -38 * gt.abs().max()
    z_err[:, 250] = 0.0  # exp of -inf is 0
    want = z.t() @ X
    err = z_err.t() @ X.abs() + 2 * U * (tokens + 2) * (z.abs().t() @ X.abs())
    assert_close(w.grad, want, err + rounded(want, DT[dtype]), "grad_weight")


def weighted_grad(tokens, vocab, dim, dtype, weights, mean=0.0, chunk=512):
    """head_grad of "none" with these weights into fp32, against float64.  Each token's
    z is held relative to its own weight for grad_hidden, and where fp16 runs out
    relative to the largest for grad_weight."""
    t = DT[dtype]
    hidden, table, targets = head_inputs(tokens, vocab, dim, dtype, sigma=0.02, know=False)
    table = (table.float() + mean).to(t)
    hidden *= 0.5
    targets[::7] = -1
    weights = weights.float().cuda()
    lse, _ = g.head_stats(hidden, table, targets)
    gx, gw = torch.full(hidden.shape, float("nan"), device="cuda"), torch.full(table.shape, float("nan"), device="cuda")
    g.head_grad(hidden, table, targets, lse, weights, grad_hidden=gx, grad_weight=gw)
    alone, _ = g.head_grad(hidden, table, targets, lse, weights, grad_hidden=torch.empty_like(gx))
    W = table.double()
    counts = targets >= 0
    most = weights[counts].abs().max().double() if bool(counts.any()) else torch.zeros((), device="cuda").double()
    want_w, err_w = torch.zeros_like(W), torch.zeros_like(W)
    out = 2.0 ** -38 if dtype == "fp16" else 0.0
    for a in range(0, tokens, chunk):
        X, y, gt = hidden[a:a + chunk].double(), targets[a:a + chunk], weights[a:a + chunk].double()
        gt = torch.where(y >= 0, gt, torch.zeros_like(gt))
        logits = X @ W.t()
        d = 2 * U * (dim + 2) * (X.abs() @ W.abs().t()) + 2 * U * logits.abs()
        want_lse = torch.logsumexp(logits, 1)
        e = d.amax(1) + (300 + 8) * U + 4 * U * (want_lse.abs() + logits.abs().amax(1))
        p = torch.exp(logits - want_lse[:, None])
        z = p.clone()
        z[torch.arange(y.numel(), device="cuda"), y.clamp(min=0)] -= 1.0
        z *= gt[:, None]
        # the product of the weight and of its scale is exact; a weight in fp32's subnormals is taken as it is
        z_err = gt.abs()[:, None] * p * (d + e[:, None] + 2.0 ** -22) + (4 * U + H[t][0]) * z.abs()
        want = z @ W
        err = (z_err + out * gt.abs()[:, None]) @ W.abs() + 2 * U * (vocab + 8) * (z.abs() @ W.abs())
        for got, what in ((gx, "with grad_weight"), (alone, "alone")):
            assert_close(got[a:a + chunk], want, err + rounded(want, torch.float32), f"grad_hidden {what} from {a}: ")
        want_w += z.t() @ X
        err_w += (z_err + out * most * (y >= 0)[:, None]).t() @ X.abs() + 2 * U * (tokens + 2) * (z.abs().t() @ X.abs())
    assert_close(gw, want_w, err_w + rounded(want_w, torch.float32), "grad_weight")
    return hidden, table, targets, weights, gx


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("mean", [0.0, 0.05])
@pytest.mark.parametrize("tokens,vocab,dim", [(1, 300, 64), (20, 50304, 64), (64, 50304, 64), (256, 1000, 72),
                                              (257, 3001, 65), (700, 50304, 40), (3000, 50304, 64)])
def test_head_weights_far_apart_keep_each_tokens_gradient(tokens, vocab, dim, mean, dtype):
    """Weights from 2^20 to 2^-20 in one call, some of them 0 or negative: every row of
    grad_hidden is as good as alone.  The largest case takes the vocabulary in pieces."""
    k = torch.arange(tokens)
    weights = torch.exp2(((k * 17) % 41 - 20).double()) * (1.0 + (k % 5) / 8.0) * torch.where(k % 3 == 0, -1.0, 1.0)
    weights[5::31] = 0.0
    weighted_grad(tokens, vocab, dim, dtype, weights, mean)


@pytest.mark.parametrize("scale", [2.0 ** 90, 2.0 ** -60])
def test_head_weights_at_the_ends_of_their_type(scale):
    k = torch.arange(40)
    weighted_grad(40, 3000, 64, "fp16", torch.exp2((-(k % 25)).double()) * scale, 0.05)


def test_head_weights_far_apart_in_16_bits_scale_rows_exactly():
    """A weight that is a power of two times another scales its row by just that, also
    from one call to the other and through the loss."""
    hidden, table, targets = head_inputs(96, 5000, 64, "fp16", sigma=0.02)
    hidden[48:], targets[48:] = hidden[:48], targets[:48]
    lse, _ = g.head_stats(hidden, table, targets)
    weights = torch.ones(96, device="cuda")
    weights[:48] = 2.0 ** -22
    gx = torch.empty(96, 64, device="cuda")
    g.head_grad(hidden, table, targets, lse, weights, grad_hidden=gx, grad_weight=torch.empty(5000, 64, device="cuda"))
    assert torch.equal(gx[:48] * 2.0 ** 22, gx[48:])
    x = hidden.detach().requires_grad_()
    up = weights * 2.0 ** 20  # the smaller ones' rows are within fp16's range too
    g.linear_cross_entropy(x, table, targets, reduction="none").backward(up)
    # the same fp32 sums times a power of two, rounded once; those from 65520 on to infinity
    assert torch.equal(x.grad, (gx * 2.0 ** 20).half())
    # none has a weight but one; weights that are no numbers stay in their rows
    weights = torch.zeros(96, device="cuda")
    weights[9] = 2.0 ** -40
    gx, _ = g.head_grad(hidden, table, targets, lse, weights, grad_hidden=torch.empty(96, 64, device="cuda"))
    assert not bool(gx[:9].any()) and not bool(gx[10:].any()) and bool(gx[9].any())
    for value in (float("inf"), float("nan")):
        weights = torch.full((96,), 2.0 ** -22, device="cuda")
        weights[3] = value
        gx, _ = g.head_grad(hidden, table, targets, lse, weights, grad_hidden=torch.empty(96, 64, device="cuda"))
        rows = torch.isfinite(gx).all(1)
        assert not bool(rows[3]) and int((~rows).sum()) == 1


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_gate8_tails_are_as_good_as_the_middle(kind, dtype):
    """act(x) and its derivative for negative x, relative to themselves down to where
    they leave the type: the exponent of a result e^-a is off by a few roundings of a <
    90, so the result by 2^-15 (gelu_tanh, with seven more roundings in a, 2^-14)."""
    t = DT[dtype]
    values = torch.cat([torch.linspace(-14.5, 0, 4001, dtype=torch.float64), torch.linspace(-88, -14.5, 1001).double()])
    x = values.cuda().to(t).view(-1, 1).contiguous().requires_grad_()  # each in a block of its own
    y = g.gate8(x, kind=kind)
    y.backward(torch.ones_like(y))
    rel = 2.0 ** (-14 if kind == "gelu_tanh" else -15)
    X = x.detach().double()
    want, _, _ = act64(X, kind)
    # e^-a below 2^-126 may be 0, which is x times as much in the result
    assert_close(y.detach(), want, rel * want.abs() + 2.0 ** -126 * X.abs() + rounded(want, t), "y")
    K = kept64(x)
    _, want, parts = act64(K, kind)  # the derivative is a sum: relative to its terms
    assert_close(x.grad, want, 2 * rel * parts + 61 * 2.0 ** -126 * K.abs() + rounded(want, t), "dx")
    f = torch.full_like(x, 0.75).detach().requires_grad_()
    y = g.gate8(x.detach(), f, kind=kind)
    y.backward(torch.ones_like(y))
    want = act64(K, kind)[0]
    assert_close(f.grad, want, rel * want.abs() + 2.0 ** -126 * K.abs() + rounded(want, t), "df")


def test_destinations_that_require_a_gradient_are_refused():
    hidden, table, targets = head_inputs(40, 100, 64, "bf16")
    lse, _ = g.head_stats(hidden, table, targets)
    one, kept = torch.ones(1, device="cuda"), g.act8_pack(hidden)
    dy = randn((40, 24), torch.bfloat16, 3)

    def made(shape):
        leaf = torch.full(shape, 5.0, device="cuda", requires_grad=True)
        return leaf, leaf * 1.0, (leaf * 1.0)[:, :]

    def grads(**into):
        return g.head_grad(hidden, table, targets, lse, one, reduction="sum", **into)

    for shape, call in (((40, 64), lambda t: grads(grad_hidden=t)), ((100, 64), lambda t: grads(grad_weight=t)),
                        ((100, 64), lambda t: grads(grad_weight=t, accumulate=True)),
                        ((24, 64), lambda t: g.linear8_grad_weight(dy, kept, t)),
                        ((24, 64), lambda t: g.linear8_grad_weight(dy, kept, t, accumulate=True)),
                        ((40, 64), lambda t: kept.unpack(out=t))):
        for t in made(shape):
            with pytest.raises(ValueError, match="requires a gradient"):
                call(t)
            assert bool((t == 5.0).all())
            with torch.no_grad():  # as torch's own writes into a parameter
                call(t.detach()), call(t)
            assert not bool((t == 5.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("grad", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("tokens,rows,cols", [(1, 8, 8), (70, 33, 50), (300, 520, 264), (3000, 64, 48), (1030, 515, 600)])
def test_linear8_grad_weight_by_itself(tokens, rows, cols, accumulate, grad, dtype):
    """Against float64, and the same bits as the layer's backward."""
    t = DT[dtype]
    x, w = randn((tokens, cols), t, 1), randn((rows, cols), t, 2, 0.05).requires_grad_()
    dy, old = randn((tokens, rows), t, 3, 0.1), randn((rows, cols), DT[grad], 4)
    K = kept64(x)
    want = dy.double().t() @ K + (old.double() if accumulate else 0.0)
    # the sum with the old value is rounded to fp32 before its type
    extra = 2 * U * (want.abs() + old.double().abs())
    err = product_error(dy.double().t(), K, want, DT[grad], extra)
    kept = g.act8_pack(x)
    alone, apart = old.clone(), padded(old.clone(), 3, 5.0)
    for into in (alone, apart):
        version = into._version
        assert g.linear8_grad_weight(dy, kept, into, accumulate=accumulate) is into and into._version > version
        assert_close(into, want, err, "grad_weight")
    assert bool((apart._base[:, cols:] == 5.0).all())
    back = old.clone()
    g.linear8(x, w, grad_weight=back, accumulate=accumulate).backward(dy)
    assert torch.equal(alone, back)


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("up", [1e-6, 65536.0, 2.0 ** -60, 2.0 ** 60])
@pytest.mark.parametrize("tokens,vocab,dim", [(64, 3000, 64), (300, 5000, 33)])
def test_head_fp16_under_loss_gradients_of_any_size(tokens, vocab, dim, up, reduction):
    """fp16 inputs: fp32 gradients scale with the loss's, and fp16 ones are those rounded."""
    hidden, table, targets = head_inputs(tokens, vocab, dim, "fp16")
    targets[::9] = -1
    counts = targets >= 0
    lse, _ = g.head_stats(hidden, table, targets)
    n = tokens if reduction == "none" else 1
    grad = torch.full((n,), up, device="cuda")
    into = [torch.full((tokens, dim), float("nan"), device="cuda"), torch.full((vocab, dim), float("nan"), device="cuda")]
    g.head_grad(hidden, table, targets, lse, grad, reduction=reduction, grad_hidden=into[0], grad_weight=into[1])
    X, W, logits, want_lse, d, e = head64(hidden, table, targets, 1.0, counts)
    gt = counts.double() * float(grad[0]) / (int(counts.sum()) if reduction == "mean" else 1)
    p = torch.exp(logits - want_lse[:, None])
    z = p.clone()
    z[torch.arange(tokens, device="cuda"), targets.clamp(min=0)] -= 1.0
    z *= gt[:, None]
    z_err = gt.abs()[:, None] * (p * (d + e[:, None] + 2.0 ** -22) + 2.0 ** -38) + (6 * U + H[torch.float16][0]) * z.abs()
    for got, a, b, z_, z_e in ((into[0], W, "grad_hidden", z, z_err), (into[1], X, "grad_weight", z.t(), z_err.t())):
        want = z_ @ a
        err = z_e @ a.abs() + 2 * U * (z_.shape[1] + 8) * (z_.abs() @ a.abs())
        assert_close(got, want, err + rounded(want, torch.float32), b)
    x, w = hidden.detach().requires_grad_(), table.detach().requires_grad_()
    g.linear_cross_entropy(x, w, targets, reduction=reduction).backward(grad.view(targets.shape if n > 1 else ()))
    assert torch.equal(x.grad, into[0].half()) and torch.equal(w.grad, into[1].half())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("tokens,vocab,dim", [(5, 300, 33), (200, 1000, 64), (300, 1003, 65), (9000, 30_000, 24)])
def test_head_grad_stays_within_its_workspace(tokens, vocab, dim, dtype):
    """The bytes that are told serve every reduction, with either gradient or both; what
    lies behind them is left alone, and what they held before does not matter."""
    hidden, table, targets = head_inputs(tokens, vocab, dim, dtype)
    targets[::5] = -1
    lse, _ = g.head_stats(hidden, table, targets)
    head = model._head(hidden, table, targets, 1.0, 0, None, 0)[1]
    L, stream = model._lib(), torch.cuda.current_stream().cuda_stream
    weights = torch.exp2((-(torch.arange(tokens, device="cuda") % 23)).float())
    for by in ((True, True), (True, False), (False, True)):
        out = [torch.empty(n, dim, device="cuda") if b else None for n, b in zip((tokens, vocab), by)]
        packed = [None if o is None else ops._matrix(o, "", None) for o in out]
        need = ctypes.c_size_t()
        assert L.gockpt_head_grad_bytes(head, *packed, ctypes.byref(need)) == 0
        ws = torch.empty(need.value + 4096, dtype=torch.uint8, device="cuda")
        assert ws.data_ptr() % 256 == 0
        for reduction, grad in ((0, weights), (1, weights[3:4].clone()), (2, weights[:1].clone())):
            got = []
            for fill in (0, 0xff):
                ws.fill_(fill)
                ws[need.value:] = 0x5a
                for o in out:
                    if o is not None:
                        o.fill_(float("nan"))
                rc = L.gockpt_head_grad(head, lse.data_ptr(), reduction, grad.data_ptr(), *packed, 0, ws.data_ptr(),
                                        need.value, stream)
                assert rc == 0, g.lib().gockpt_last_error(None)
                assert bool((ws[need.value:] == 0x5a).all())
                got.append([o.clone() for o in out if o is not None])
            for a, b in zip(*got):
                assert torch.equal(a, b) and bool(torch.isfinite(a).all())


@pytest.mark.parametrize("tokens", [40, 300])
def test_head_weights_far_apart_replay_from_a_graph(tokens):
    """fp16 with a weight for each token, captured: replays with other weights are the eager calls."""
    hidden, table, targets = head_inputs(tokens, 3000, 64, "fp16")
    weights, into = torch.ones(tokens, device="cuda"), torch.zeros(3000, 64, device="cuda")
    x = hidden.detach().requires_grad_()
    w = table.detach().requires_grad_()

    def run():
        x.grad = None
        loss = g.linear_cross_entropy(x, w, targets, reduction="none", grad_weight=into)
        loss.backward(weights)
        return x.grad, into

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            run()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for k in range(4):
        weights.copy_(torch.exp2((-(torch.arange(tokens, device="cuda") * (k + 1) % 25)).float()))
        targets.copy_(torch.roll(targets, 1))
        targets[k] = -1
        for t in captured:
            t.fill_(float("nan"))
        graph.replay()
        got = [t.clone() for t in captured]
        torch.cuda.synchronize()
        lse, _ = g.head_stats(hidden, table, targets)
        want = g.head_grad(hidden, table, targets, lse, weights, grad_weight=torch.zeros_like(into))
        for a, b in zip(got, want):
            assert torch.equal(a, b), k


def test_head_weights_far_apart_over_ranks():
    """Ranks that split the vocabulary, in fp16 with a weight for each token: their parts
    of grad_hidden add up to what one rank has, their rows of grad_weight are its rows."""
    tokens, vocab, dim = 300, 5000, 64
    hidden, table, targets = head_inputs(tokens, vocab, dim, "fp16", sigma=0.02)
    targets[::6] = -1
    weights = torch.exp2((-(torch.arange(tokens, device="cuda") % 25)).float())
    lse, _ = g.head_stats(hidden, table, targets)
    want = g.head_grad(hidden, table, targets, lse, weights, grad_hidden=torch.empty(tokens, dim, device="cuda"),
                       grad_weight=torch.empty(vocab, dim, device="cuda"))
    total = torch.zeros(tokens, dim, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(total)
    for a, b in ((0, 1700), (1700, 1703), (1703, 5000)):
        gx, gw = g.head_grad(hidden, table[a:b], targets, lse, weights, first_id=a, classes=vocab,
                             grad_hidden=torch.empty(tokens, dim, device="cuda"),
                             grad_weight=torch.empty(b - a, dim, device="cuda"))
        total += gx
        # the same terms in another order, and other classes' two first tokens: by the sums' errors and z's halves
        p = torch.exp(hidden.double() @ table[a:b].double().t() - lse.double()[:, None])
        size += weights[:, None].double() * (p @ table[a:b].double().abs())
        z = p * (targets >= 0)[:, None] * weights[:, None]
        at = (targets >= a) & (targets < b)
        z[at.nonzero()[:, 0], targets[at] - a] -= weights[at]
        err = (2.0 ** -11 * z.abs() + 2.0 ** -38).t() @ hidden.double().abs()
        err += 4 * U * (tokens + 2) * (z.abs().t() @ hidden.double().abs())
        assert_close(gw, want[1][a:b].double(), 2 * err, f"grad_weight from {a}")
    own = weights[:, None].double() * table[targets.clamp(min=0)].double().abs()
    err = 2.0 ** -10 * size + 2.0 ** -37 * weights[:, None].double() * table.double().abs().sum(0)
    err += 4 * U * (vocab + 8) * (size + own)
    assert_close(total, want[0].double(), err, "grad_hidden")
