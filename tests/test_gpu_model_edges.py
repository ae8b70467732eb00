"""Edges of the model's operators on the GPU.  Tolerances as in test_gpu_model,
whose helpers these tests take."""
import copy
import math
import pickle

import pytest

import paper_2511_07035_amd as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_model import DT, H, U, assert_close, head_inputs, kept64, product_error, randn, rounded  # noqa: E402


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
