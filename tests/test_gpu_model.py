"""The head's cross entropy, 8-bit activations, the linear layer and the
activation that keep them, on the GPU, against plain implementations in float64.

Tolerances, with u = 2^-24 (a rounding to fp32) and h half a step of the
output's type, relative to the value:
  act8      exact.
  linear8   products of 16-bit values are exact in fp32; the sum of n of them,
            in whichever order, is off by n 2u sum|terms| at most (2u a step:
            the matrix cores may truncate), then h of the result.
  loss      a logit is off by d = (n + 2) 2u |scale| sum|x w|; the log of the sum
            of exp by as much (the most of any class), and by the errors of the
            sum itself: exp2 and its argument 4u and |l| u each, the additions
            300 u in all (128 in a lane, then by halves); logs and products 4u of
            what they give.
  gradients z is off by g p (e + 2^-22), e the error of its exponent (logit and
            lse), and by half a step hz of the 16-bit type (2^-38 |g| where fp16
            runs out); the products take both times |w| or |x|, with the sums'
            n 2u sum|terms| and h of the result.
  gate8     16-bit types take exp2 and a reciprocal of the hardware, off by
            |x| u + 4u: 2^-17 for all |x| < 88, where anything is left of the
            result; the normal distribution's tail by 1.5e-7 |x|.  fp32: library
            functions within 8u, 16 u for the few products of a result.  The
            argument of erfc is -x / sqrt 2 with the constant and the product
            rounded, 2u in all; erfc(a) falls as exp(-a^2), so that is a 2 a 2u a
            = 2 x^2 u of it; the argument of exp(-x^2 / 2) is rounded twice, x^2 u
            of the result.  Where exp(-x) leaves fp32's range (x < -88, or the
            product that gelu_tanh puts in its place) 1 / (1 + exp(-x)) is 0 for
            less than 2^-126: |x| 2^-126 of the result, and that times the inner
            slope, at most |x| 60 there, of the derivative.
"""
import math

import pytest

import paper_2511_07035_amd as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
H = {torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float16: (2.0 ** -11, 2.0 ** -25),
     torch.float32: (U, 2.0 ** -150)}


def randn(shape, dtype, seed, sigma=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.empty(shape, device="cuda").normal_(0.0, sigma, generator=gen).to(dtype)


def rounded(want, dtype):
    """Half a step of dtype at want, in float64."""
    rel, least = H[dtype]
    return want.abs() * rel + least


def assert_close(got, want, err, what=""):
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got.double() - want).abs() <= err)
    if bool(bad.any()):
        i = tuple(x[0].item() for x in bad.nonzero(as_tuple=True))
        raise AssertionError(f"{what}{list(i)}: {got[i].item()} for {want[i].item()}, off by "
                             f"{abs(got[i].double().item() - want[i].item()):.3g}, allowed {err[i].item():.3g}; "
                             f"{int(bad.sum())} of {bad.numel()}")


def padded(t, extra, fill=float("nan")):
    """t as the left columns of a wider buffer."""
    wide = torch.full((*t.shape[:-1], t.shape[-1] + extra), fill, dtype=t.dtype, device=t.device)
    wide[..., :t.shape[-1]] = t
    return wide[..., :t.shape[-1]]


def shifted(t, by=1):
    """t contiguous, but `by` elements behind an aligned address."""
    buf = torch.zeros(t.numel() + by, dtype=t.dtype, device=t.device)
    out = buf[by:].view(t.shape)
    out.copy_(t)
    return out


# ---- 8 bits ----------------------------------------------------------------------


def kept64(x):
    """What x stands for in 8 bits, in float64, from the definition."""
    cols = x.shape[-1]
    v = x.detach().double().reshape(-1, cols) if x.numel() else x.double().reshape(math.prod(x.shape[:-1]), cols)
    out = torch.empty_like(v)
    most_of = {torch.float16: 65504.0, torch.bfloat16: 3.3895313892515355e38, torch.float32: 3.4028234663852886e38}
    for a in range(0, cols, 32):
        b = v[:, a:a + 32]
        top = b.abs().amax(1, keepdim=True)
        _, e = torch.frexp(top / 127.0)  # in [2^(e-1), 2^e)
        e = e.double()
        e = torch.where(127.0 * torch.exp2(e - 1) >= top, e - 1, e).clamp(min=-126)
        c = torch.round(b * torch.exp2(-e))
        c = torch.where(c.abs() * torch.exp2(e) > most_of[x.dtype], c.sign() * 63, c)
        out[:, a:a + 32] = torch.where(torch.isfinite(top), c * torch.exp2(e), torch.full_like(c, float("nan")))
    return out.view(x.shape)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shape", [(1, 1), (1, 31), (3, 32), (5, 33), (7, 64), (2, 3, 95), (130, 1157), (64, 4096), (1000, 7)])
def test_act8(shape, dtype):
    x = randn(shape, DT[dtype], 3)
    x.view(-1)[::17] *= 30
    a = g.act8_pack(x)
    want = kept64(x)
    got = a.unpack()
    assert got.dtype == x.dtype and got.shape == x.shape
    assert torch.equal(got.double(), want)
    blocks = -(-shape[-1] // 32)
    assert a.codes.shape == (x.numel() // shape[-1], 32 * blocks) and a.scales.shape == (x.numel() // shape[-1], blocks)
    assert int(a.codes.to(torch.int16).abs().max()) <= 127
    assert not bool(a.codes[:, shape[-1]:].any())  # zeros behind the last column
    # from rows apart and at odd addresses, and into both; over what is there
    for y in (padded(x, 5), shifted(x), padded(x, 64)):
        b = g.act8_pack(y, out=g.act8_pack(torch.ones_like(x)))
        assert torch.equal(b.codes, a.codes) and torch.equal(b.scales, a.scales)
    for out in (padded(torch.zeros_like(x), 3, 7.0), shifted(torch.zeros_like(x))):
        a.unpack(out=out)
        assert torch.equal(out.double(), want)
        if out._base is not None and out._base.shape[-1] == shape[-1] + 3:
            assert bool((out._base[..., shape[-1]:] == 7.0).all())
    if dtype != "fp32":
        assert torch.equal(a.unpack(dtype=torch.float32).double(), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_act8_at_the_ends_of_a_type(dtype):
    t = DT[dtype]
    info = torch.finfo(t)
    rows = [[info.max, -info.max, 1.0], [info.max * 0.99, info.max * 0.3], [info.tiny, -info.tiny, info.tiny / 2],
            [info.smallest_normal, 0.0], [0.0, -0.0], [127.0, 126.5, 0.5, 1.5, 2.5, -63.5], [127.5, 64.0, 0.5, 1.5],
            [128.0, 1.0, 3.0, 5.0], [63.5, 0.25, 0.75], [1.984375, 0.0078125], [65024.0, 256.0], [65056.0, 512.0]]
    x = torch.zeros(len(rows), 40, device="cuda", dtype=t)
    for i, r in enumerate(rows):
        x[i, :len(r)] = torch.tensor(r, dtype=torch.float64).to(t)
        x[i, 33] = x[i, 0]
    a = g.act8_pack(x)
    got = a.unpack().double()
    assert torch.equal(got, kept64(x))
    assert bool(torch.isfinite(got).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_act8_of_what_is_no_number(dtype, value):
    x = randn((4, 100), DT[dtype], 5)
    x[1, 40] = value
    x[3, 99] = value
    a = g.act8_pack(x)
    assert int((a.scales == 255).sum()) == 2
    got, want = a.unpack().double(), kept64(x)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    assert bool(torch.isnan(got[1, 32:64]).all()) and bool(torch.isnan(got[3, 96:]).all())


def test_act8_without_elements():
    for shape in ((0, 8), (5, 0), (0,), (3, 0, 7)):
        a = g.act8_pack(torch.zeros(shape, device="cuda"))
        assert a.unpack().shape == torch.Size(shape) and a.nbytes >= 0


def test_act8_beyond_32_bits():
    x = torch.zeros(70_000, 32_768, dtype=torch.float16, device="cuda")
    tail = randn((3, 32_768), torch.float16, 8)
    x[-3:] = tail
    a = g.act8_pack(x)
    assert torch.equal(a.codes[-3:], g.act8_pack(tail).codes) and not bool(a.codes[-5:-3].any())
    assert torch.equal(a.unpack()[-3:], g.act8_pack(tail).unpack())


def test_act8_writes_nothing_else():
    x = randn((9, 70), torch.bfloat16, 4)
    buf = torch.full((20, 70), 3.0, dtype=torch.bfloat16, device="cuda")
    g.act8_pack(x).unpack(out=buf[5:14])
    assert bool((buf[:5] == 3.0).all()) and bool((buf[14:] == 3.0).all())


# ---- linear layer -----------------------------------------------------------------


def product_error(a, b, want, dtype, extra=0.0):
    """Of a @ b (float64) as a product kernel gives it in dtype."""
    return 2 * U * (a.shape[1] + 2) * (a.abs() @ b.abs()) + rounded(want, dtype) + extra


LINEAR = [(1, 1, 1), (1, 8, 8), (1, 4096, 512), (2, 100, 33), (7, 64, 176), (31, 40, 64), (32, 128, 256), (33, 130, 72),
          (96, 176, 64), (129, 257, 65), (200, 1000, 136), (255, 256, 64), (257, 264, 128), (300, 77, 1157),
          (513, 320, 520), (1000, 48, 2000), (40, 3000, 40), (5000, 24, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("tokens,rows,cols", LINEAR)
def test_linear8(tokens, rows, cols, dtype):
    t = DT[dtype]
    x, w = randn((tokens, cols), t, 1).requires_grad_(), randn((rows, cols), t, 2, 0.05).requires_grad_()
    dy = randn((tokens, rows), t, 3)
    y = g.linear8(x, w)
    y.backward(dy)
    X, W, D = x.detach().double(), w.detach().double(), dy.double()
    want = X @ W.t()
    assert y.dtype == t
    assert_close(y.detach(), want, product_error(X, W.t(), want, t), "y")
    want = D @ W
    assert_close(x.grad, want, product_error(D, W, want, t), "dx")
    K = kept64(x)
    want = D.t() @ K
    assert_close(w.grad, want, product_error(D.t(), K, want, t), "dw")
    # without gradients: the same output, on another stream too
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = g.linear8(x.detach(), w.detach(), stream=s)
    s.synchronize()
    assert torch.equal(other, y.detach())


@pytest.mark.parametrize("dtype,tokens,rows,cols", [("bf16", 4100, 4104, 4200), ("fp16", 3999, 4133, 4331),
                                                    ("bf16", 2111, 3090, 1160), ("fp16", 20_001, 130, 72)])
def test_linear8_of_many_tiles(dtype, tokens, rows, cols):
    """Large tiles, with edges in every direction, and sums long enough that
    blocks take them in turn; into fp32 as well."""
    t = DT[dtype]
    x, w = randn((tokens, cols), t, 1).requires_grad_(), randn((rows, cols), t, 2, 0.05).requires_grad_()
    dy = randn((tokens, rows), t, 3)
    into = randn((rows, cols), torch.float32, 4)
    old = into.double().clone()
    y = g.linear8(x, w, grad_weight=into, accumulate=True)
    y.backward(dy)
    X, W, D = x.detach().double(), w.detach().double(), dy.double()
    want = X @ W.t()
    assert_close(y.detach(), want, product_error(X, W.t(), want, t), "y")
    want = D @ W
    assert_close(x.grad, want, product_error(D, W, want, t), "dx")
    K = kept64(x)
    want = D.t() @ K + old
    extra = 2 * U * (want.abs() + old.abs())
    assert_close(into, want, product_error(D.t(), K, want, torch.float32, extra), "dw")


@pytest.mark.parametrize("grad", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("tokens,rows,cols", [(1, 8, 8), (70, 33, 50), (300, 520, 264), (3000, 64, 48)])
def test_linear8_gradient_into_a_buffer(tokens, rows, cols, accumulate, grad):
    for dtype in ("bf16", "fp16"):
        t = DT[dtype]
        x, w = randn((tokens, cols), t, 1), randn((rows, cols), t, 2, 0.05).requires_grad_()
        dy = randn((tokens, rows), t, 3, 0.1)
        buf = torch.full((rows + 2, cols + 3), 5.0, dtype=DT[grad], device="cuda")
        into = buf[1:-1, 1:-2]
        into.copy_(randn((rows, cols), DT[grad], 4))
        old = into.double().clone()
        version = into._version
        g.linear8(x, w, grad_weight=into, accumulate=accumulate).backward(dy)
        assert w.grad is None and into._version > version
        K = kept64(x)
        want = dy.double().t() @ K + (old if accumulate else 0.0)
        # the sum with the old value is rounded to fp32 before its type
        extra = 2 * U * (want.abs() + old.abs())
        assert_close(into, want, product_error(dy.double().t(), K, want, DT[grad], extra), "dw")
        for edge in (buf[0], buf[-1], buf[:, 0], buf[:, -2:]):
            assert bool((edge == 5.0).all())
        # the call alone gives the same
        into.copy_(old)
        keep = g.act8_pack(x)
        alone = into.clone()
        g.linear8_grad_weight(dy, keep, alone, accumulate=accumulate)
        again = into.clone()
        g.linear8_grad_weight(dy, keep, again, accumulate=accumulate)
        assert torch.equal(alone, again)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_linear8_strides(dtype):
    t = DT[dtype]
    base_x, base_w, base_d = randn((60, 72), t, 1), randn((136, 72), t, 2), randn((60, 136), t, 3)
    want = None
    for px, pw, pd in ((lambda a: a,) * 3, (lambda a: padded(a, 8),) * 3, (lambda a: padded(a, 5),) * 3,
                       (shifted,) * 3, (lambda a: shifted(a, 8),) * 3, (lambda a: a.t().contiguous().t(), shifted, lambda a: padded(a, 1))):
        x, w = px(base_x).detach().requires_grad_(), pw(base_w).detach().requires_grad_()
        y = g.linear8(x, w)
        y.backward(pd(base_d))
        got = (y.detach(), x.grad, w.grad)
        if want is None:
            want = got
        for a, b in zip(got, want):  # the same sums, wherever the inputs lie
            assert torch.equal(a, b)
    # more dimensions, rows apart; an expanded gradient
    x = padded(base_x, 8).view(4, 15, 72).detach().requires_grad_()
    w = base_w.detach().requires_grad_()
    y = g.linear8(x, w)
    assert y.shape == (4, 15, 136) and torch.equal(y.detach().view(60, 136), want[0])
    y.sum().backward()
    ones = torch.ones(60, 136, dtype=torch.float64, device="cuda")
    dx = ones @ base_w.double()
    assert_close(x.grad.view(60, 72), dx, product_error(ones, base_w.double(), dx, t))


def test_linear8_offsets_beyond_32_bits():
    for cols in (64, 50):
        big = torch.zeros(3, (1 << 31) + 64, dtype=torch.bfloat16, device="cuda")[:, :cols]
        big.copy_(randn((3, cols), torch.bfloat16, 1))
        w = randn((40, cols), torch.bfloat16, 2)
        x = big.clone().requires_grad_()
        assert torch.equal(g.linear8(big, w), g.linear8(x, w).detach())
        grad = torch.zeros(3, (1 << 31) + 64, dtype=torch.bfloat16, device="cuda")[:, :40]
        grad.copy_(randn((3, 40), torch.bfloat16, 3))
        a, b = torch.zeros(40, cols, device="cuda"), torch.zeros(40, cols, device="cuda")
        g.linear8_grad_weight(grad, g.act8_pack(big), a)
        g.linear8_grad_weight(grad.clone(), g.act8_pack(x), b)
        assert torch.equal(a, b)
        del big, grad


def test_linear8_empty():
    w = randn((5, 8), torch.bfloat16, 1).requires_grad_()
    x = torch.zeros(0, 8, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    y = g.linear8(x, w)
    assert y.shape == (0, 5)
    y.backward(torch.zeros_like(y))
    assert x.grad.shape == (0, 8) and bool((w.grad == 0).all())
    into = torch.full((5, 8), 2.0, device="cuda")
    g.linear8(x, w, grad_weight=into, accumulate=True).backward(torch.zeros_like(y))
    assert bool((into == 2.0).all())
    # no columns: sums of nothing
    x = torch.zeros(3, 0, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    w = torch.zeros(5, 0, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    y = g.linear8(x, w)
    assert y.shape == (3, 5) and bool((y == 0).all())
    y.backward(torch.ones_like(y))
    assert x.grad.shape == (3, 0) and w.grad.shape == (5, 0)
    # no outputs: no gradient of x
    x = torch.ones(3, 8, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    w = torch.zeros(0, 8, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    y = g.linear8(x, w)
    assert y.shape == (3, 0)
    y.backward(torch.zeros_like(y))
    assert bool((x.grad == 0).all()) and w.grad.shape == (0, 8)


def test_linear8_keeps_little_and_only_what_it_needs():
    x, w = randn((256, 512), torch.bfloat16, 1).requires_grad_(), randn((64, 512), torch.bfloat16, 2)
    y = g.linear8(x, w)
    assert y.grad_fn.kept is None  # the weight needs no gradient
    y.backward(torch.ones_like(y))
    w = w.requires_grad_()
    y = g.linear8(x.detach(), w)
    assert y.grad_fn.kept.nbytes == 256 * 512 * 33 // 32
    assert [t is None for t in y.grad_fn.saved_tensors] == [True, False]
    y.backward(torch.ones_like(y), retain_graph=True)
    first = w.grad.clone()
    y.backward(torch.ones_like(y))
    assert torch.equal(w.grad, first + first)
    with pytest.raises(RuntimeError):  # freed
        y.backward(torch.ones_like(y))


def test_graphs_let_go_of_what_they_keep():
    """A result that lives on after the backward holds none of the 8-bit copies, and hooks may move them."""
    x, w = randn((512, 1024), torch.bfloat16, 1).requires_grad_(), randn((256, 1024), torch.bfloat16, 2).requires_grad_()
    f = randn((512, 256), torch.bfloat16, 3).requires_grad_()

    def run():
        x.grad = w.grad = f.grad = None
        return g.gate8(g.linear8(x, w), f)
    y = run()
    y.backward(f.detach())
    want = x.grad.clone(), w.grad.clone(), f.grad.clone()
    del y
    x.grad = w.grad = f.grad = None
    before = torch.cuda.memory_allocated()
    y = run()
    held = torch.cuda.memory_allocated() - before
    assert held >= 33 * (512 * 1024 + 2 * 512 * 256) // 32
    y.backward(f.detach())
    held = torch.cuda.memory_allocated() - before - 2 * (x.numel() + w.numel() + f.numel())
    assert held <= 2 * y.numel() + 3 * 512, held  # y itself
    with pytest.raises(RuntimeError):
        y.backward(f.detach())
    with torch.autograd.graph.save_on_cpu():
        y = run()
    y.backward(f.detach())
    for got, one in zip((x.grad, w.grad, f.grad), want):
        assert torch.equal(got, one)


def test_linear8_of_infinities():
    x = randn((40, 96), torch.bfloat16, 1)
    x[3, 70] = float("inf")
    w = randn((24, 96), torch.bfloat16, 2).requires_grad_()
    y = g.linear8(x, w)
    assert int((~torch.isfinite(y)).any(1).sum()) == 1
    y.backward(torch.ones_like(y))
    bad = ~torch.isfinite(w.grad)
    assert bool(bad[:, 64:].all()) and not bool(bad[:, :64].any())  # the block's columns tell


# ---- activation -----------------------------------------------------------------------


def act64(x, kind):
    if kind == "silu":
        s = torch.sigmoid(x)
        return x * s, s * (1 + x * (1 - s)), s.abs() + (x * s * (1 - s)).abs()
    if kind == "gelu":
        c, p = 0.5 * torch.erfc(-x / math.sqrt(2)), torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
        return x * c, c + x * p, c + (x * p).abs()
    a, b = 2 * math.sqrt(2 / math.pi), 0.044715
    s = torch.sigmoid(a * (x + b * x ** 3))
    d = x * s * (1 - s) * a * (1 + 3 * b * x * x)
    return x * s, s + d, s + d.abs()


def act_errors(x, kind, dtype):
    """Of act and of its derivative, before rounding."""
    y, d, parts = act64(x, kind)
    gone = 2.0 ** -126 * x.abs()
    if dtype == torch.float32:
        more = torch.zeros_like(x)
        if kind == "gelu":
            more = 2 * U * x * x
        elif kind == "gelu_tanh":
            # the exponent is a product of rounded sums: off by 6u of it
            more = 6 * U * 1.6 * x.abs() * (1 + 0.045 * x * x)
        return y.abs() * (16 * U + more) + gone, parts * (16 * U + 2 * more * (1 + x.abs())) + 61 * gone
    far = 1 + (x.abs().clamp(max=8) if kind == "gelu_tanh" else 0)
    tail = 1.6e-7 if kind == "gelu" else 0.0
    return 2.0 ** -16 * y.abs() * far + tail * x.abs() + gone, 2.0 ** -16 * parts * far + tail + 61 * gone


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape", [(1, 1), (3, 31), (2, 32), (5, 77), (2, 3, 176), (300, 1024), (1501, 85)])
def test_gate8(shape, gated, kind, dtype):
    t = DT[dtype]
    x = randn(shape, t, 1, 2.0)
    x.view(-1)[::13] *= 5
    x = x.requires_grad_()
    f = randn(shape, t, 2).requires_grad_() if gated else None
    dy = randn(shape, t, 3)
    y = g.gate8(x, f, kind=kind)
    y.backward(dy)
    X, D = x.detach().double(), dy.double()
    F = f.detach().double() if gated else torch.ones_like(X)
    a, _, _ = act64(X, kind)
    err, _ = act_errors(X, kind, t)
    want = a * F
    assert y.dtype == t
    assert_close(y.detach(), want, err * F.abs() + 2 * U * want.abs() + rounded(want, t), "y")
    K, G = kept64(x), kept64(f) if gated else torch.ones_like(X)
    a, d, _ = act64(K, kind)
    err_a, err_d = act_errors(K, kind, t)
    want = D * d * G
    assert_close(x.grad, want, (D * G).abs() * err_d + 4 * U * want.abs() + rounded(want, t), "dx")
    if gated:
        want = D * a
        assert_close(f.grad, want, D.abs() * err_a + 2 * U * want.abs() + rounded(want, t), "df")
    # without gradients, and where inputs lie apart: the same bits
    for X2, F2 in ((x.detach(), f.detach() if gated else None),
                   (padded(x.detach(), 3), padded(f.detach(), 8) if gated else None),
                   (shifted(x.detach()), shifted(f.detach(), 3) if gated else None)):
        assert torch.equal(g.gate8(X2, F2, kind=kind), y.detach())


def test_gate8_halves_of_one_buffer_and_one_needed_gradient():
    both = randn((6, 7, 2 * 90), torch.bfloat16, 1).requires_grad_()
    y = g.gate8(both[..., :90], both[..., 90:])
    y.backward(torch.ones_like(y))
    x, f = both.detach()[..., :90].clone().requires_grad_(), both.detach()[..., 90:].clone().requires_grad_()
    y2 = g.gate8(x, f)
    y2.sum().backward()  # an expanded gradient
    assert torch.equal(y.detach(), y2.detach())
    assert torch.equal(both.grad, torch.cat([x.grad, f.grad], -1))
    for only in (0, 1):
        a, b = x.detach().requires_grad_(only == 0), f.detach().requires_grad_(only == 1)
        g.gate8(a, b).sum().backward()
        assert torch.equal((a, b)[only].grad, (x, f)[only].grad) and (a, b)[1 - only].grad is None
    # the same tensor twice: both gradients add up
    z = x.detach().requires_grad_()
    g.gate8(z, z).sum().backward()
    u, v = z.detach().requires_grad_(), z.detach().requires_grad_()
    g.gate8(u, v).sum().backward()
    assert torch.equal(z.grad, u.grad + v.grad)


@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_gate8_far_out(kind, dtype):
    x = torch.tensor([[1e30, -1e30, 100.0, -100.0, 40.0, -40.0, 0.0, -0.0, 88.0, -88.0, 1e4, -1e4]], device="cuda")
    x = x.to(DT[dtype]).repeat(1, 3).t().contiguous().requires_grad_()  # each in a block of its own
    y = g.gate8(x, kind=kind)
    y.backward(torch.ones_like(y))
    X = x.detach().double()
    a = torch.where(X > 30, X, torch.where(X < -30, torch.zeros_like(X), act64(X, kind)[0]))
    assert_close(y.detach(), a, rounded(a, DT[dtype]) + 1e-12)
    d = torch.where(X > 30, torch.ones_like(X), torch.where(X < -30, torch.zeros_like(X), act64(X, kind)[1]))
    assert_close(x.grad, d, rounded(d, DT[dtype]) + 1e-12)


@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_gate8_gradient_against_differences(kind):
    # inputs that 8 bits hold exactly: the gradient is the function's own
    x = g.act8_pack(randn((4, 64), torch.float32, 1)).unpack()
    f = g.act8_pack(randn((4, 64), torch.float32, 2)).unpack()
    x, f, dy = x.requires_grad_(), f.requires_grad_(), randn((4, 64), torch.float32, 3)
    g.gate8(x, f, kind=kind).backward(dy)
    step = 1e-4

    def total(a, b):
        return act64(a, kind)[0] * b * dy.double()

    X, F = x.detach().double(), f.detach().double()
    # a central difference is off by step^2 / 6 of a third derivative, below 2 here, times |f dy|
    near = (total(X + step, F) - total(X - step, F)) / (2 * step)
    assert bool(((x.grad.double() - near).abs() <= step ** 2 * (F * dy).abs() + 32 * U * (F * dy).abs() + 1e-10).all())
    near = (total(X, F + step) - total(X, F - step)) / (2 * step)
    assert bool(((f.grad.double() - near).abs() <= 32 * U * dy.double().abs() * (1 + X.abs()) + 1e-10).all())


# ---- the head's cross entropy -----------------------------------------------------------


def head64(hidden, table, targets, scale, counts):
    """Logits, lse, losses in float64, and the errors of logit and lse."""
    X, W = hidden.double(), table.double()
    X = torch.where(counts[:, None], X, torch.zeros_like(X))
    logits = scale * (X @ W.t())
    d = 2 * U * (X.shape[1] + 2) * abs(scale) * (X.abs() @ W.abs().t()) + 2 * U * logits.abs()
    lse = torch.logsumexp(logits, 1)
    e = d.amax(1) + (300 + 8) * U + 4 * U * (lse.abs() + logits.abs().amax(1))
    return X, W, logits, lse, d, e


def head_check(hidden, table, targets, *, scale=1.0, reduction="mean", first_id=0, ignore_id=None, up=1.0, grad=None,
               accumulate=False):
    """The loss and both gradients of one call against float64."""
    t, n = hidden.dtype, targets.numel()
    y = targets.reshape(-1) - first_id
    counts = (y >= 0) & (y < table.shape[0])
    if ignore_id is not None:
        counts &= targets.reshape(-1) != ignore_id
    flat = hidden.reshape(n, -1) if n else hidden.reshape(0, table.shape[1])
    X, W, logits, lse, d, e = head64(flat, table, y, scale, counts)
    at = y.clamp(min=0, max=table.shape[0] - 1)
    own = logits.gather(1, at[:, None])[:, 0]
    each = torch.where(counts, lse - own, torch.zeros_like(lse))
    each_err = torch.where(counts, 2 * e, torch.zeros_like(lse))
    kept = int(counts.sum())
    per = 1.0 / max(kept, 1) if reduction == "mean" else 1.0
    h, w = hidden.detach().requires_grad_(), table.detach().requires_grad_()
    into = None
    if grad is not None:
        into = randn(table.shape, DT[grad], 77)
        old = into.double().clone()
    loss = g.linear_cross_entropy(h, w, targets, scale=scale, reduction=reduction, first_id=first_id,
                                  ignore_id=ignore_id, grad_weight=into, accumulate=accumulate)
    assert loss.dtype == torch.float32
    if reduction == "none":
        assert_close(loss.detach().reshape(-1), each, each_err, "loss")
        weights = randn(targets.shape, torch.float32, 9) * up
        loss.backward(weights)
        gt = weights.reshape(-1).double()
    else:
        total = each.sum() * per
        assert loss.shape == ()
        assert abs(loss.item() - total.item()) <= float(each_err.sum() * per + U * each.abs().sum() * per), (loss.item(), total.item())
        loss.backward(torch.full((), up, device="cuda"))
        gt = torch.full((n,), up * per, dtype=torch.float64, device="cuda")
    gt = torch.where(counts, gt, torch.zeros_like(gt))
    p = torch.exp(logits - lse[:, None])
    z = p.clone()
    z[torch.arange(n, device="cuda"), at] -= 1.0
    z *= gt[:, None]
    hz = H[t][0]
    z_err = gt.abs()[:, None] * p * (d + e[:, None] + 2.0 ** -22) + 4 * U * z.abs() + hz * z.abs() + \
        2.0 ** -38 * gt.abs().max().clamp(min=0) if n else z
    W1, X1 = W.abs(), X.abs()
    if n:
        want = scale * (z @ W)
        err = abs(scale) * (z_err @ W1 + 2 * U * (W.shape[0] + 8) * (z.abs() @ W1)) + rounded(want, t)
        assert_close(h.grad.reshape(n, -1), want, err, "grad_hidden")
    assert h.grad.shape == hidden.shape
    want = scale * (z.t() @ X)
    out = w.grad if into is None else into
    err = abs(scale) * (z_err.t() @ X1 + 2 * U * (n + 2) * (z.abs().t() @ X1))
    if accumulate:
        want = want + old
        err = err + 2 * U * (old.abs() + want.abs())
    assert_close(out, want, err + rounded(want, out.dtype), "grad_weight")
    if into is not None:
        assert w.grad is None
    return loss.detach(), h.grad, out


def head_inputs(tokens, vocab, dim, dtype, seed=1, sigma=0.1, know=True):
    t = DT[dtype]
    table = randn((vocab, dim), t, seed, sigma)
    hidden = randn((tokens, dim), t, seed + 1)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 2)
    targets = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    if know and tokens:
        boost = 8 * torch.rand(tokens, 1, generator=gen, device="cuda") / (sigma * sigma * dim)
        hidden += (boost * table[targets].float()).to(t)
    return hidden, table, targets


HEAD = [(1, 1, 1), (1, 7, 8), (1, 32000, 64), (2, 300, 33), (31, 129, 64), (32, 256, 72), (33, 257, 40), (96, 320, 64),
        (100, 1000, 130), (129, 127, 256), (257, 2000, 65), (300, 50, 1157), (520, 777, 136), (1000, 4099, 48)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("tokens,vocab,dim", HEAD)
def test_head(tokens, vocab, dim, dtype):
    hidden, table, targets = head_inputs(tokens, vocab, dim, dtype)
    head_check(hidden, table, targets)
    targets[::3] = -1
    head_check(hidden, table, targets, reduction="sum", up=0.5)
    head_check(hidden, table, targets.int(), reduction="none", scale=0.5, grad="fp32", accumulate=True)


@pytest.mark.parametrize("dtype,dim", [("bf16", 520), ("fp16", 523)])
def test_head_of_many_tiles(dtype, dim):
    hidden, table, targets = head_inputs(1500, 9001, dim, dtype)
    targets[7::11] = -1
    targets[0], targets[1] = 0, 9000
    head_check(hidden, table, targets, up=1024.0)
    head_check(hidden, table, targets, reduction="none", scale=-0.25, grad="fp32", accumulate=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("tokens,vocab,dim", [(9, 40, 24), (1024, 600, 40), (1025, 3001, 72), (3000, 1100, 264)])
def test_head_targets_keep_what_rounding_took(tokens, vocab, dim, dtype):
    """Neither grad_hidden nor the grad_weight rows of classes with up to two tokens have the half step that
    z at the target is rounded by: their tolerance counts it for the other terms only."""
    hidden, table, targets = head_inputs(tokens, vocab, dim, dtype, know=False)
    targets[5::7] = -1
    counts = targets >= 0
    kept, n = counts.nonzero()[:, 0], int(counts.sum())
    X, W, logits, lse, d, e = head64(hidden[kept], table, targets[kept], 1.0, counts[kept])
    h, w = hidden.requires_grad_(), table.requires_grad_()
    g.linear_cross_entropy(h, w, targets, reduction="sum").backward()
    p = torch.exp(logits - lse[:, None])
    own = torch.nn.functional.one_hot(targets[kept], vocab).double()
    z = p - own
    err = p * (d + e[:, None] + 2.0 ** -22) + 8 * U * z.abs() + H[DT[dtype]][0] * p * (1 - own) + 2.0 ** -38
    want = z @ W
    assert_close(h.grad[kept], want, err @ W.abs() + 2 * U * (vocab + 8) * (z.abs() @ W.abs()) + rounded(want, h.dtype),
                 "grad_hidden")
    few = (own.sum(0) > 0) & (own.sum(0) <= 2)
    assert int(few.sum()) > 3
    want = z.t() @ X
    err = err.t() @ X.abs() + 2 * U * (n + 8) * (z.abs().t() @ X.abs()) + rounded(want, w.dtype)
    assert_close(w.grad[few], want[few], err[few], "grad_weight")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("tokens,vocab,dim", [(40, 500, 64), (300, 700, 72), (5, 100, 33)])
def test_head_masks(tokens, vocab, dim, dtype):
    hidden, table, targets = head_inputs(tokens, vocab, dim, dtype)
    targets[0] = 0
    targets[-1] = vocab - 1
    for kind in ("first", "last", "all but one", "all", "beyond", "ignored"):
        y, x, ignore = targets.clone(), hidden.clone(), None
        if kind == "first":
            gone = torch.arange(tokens, device="cuda") < tokens // 2
        elif kind == "last":
            gone = torch.arange(tokens, device="cuda") > 2
        elif kind == "all but one":
            gone = torch.arange(tokens, device="cuda") != tokens // 2
        elif kind == "all":
            gone = torch.ones(tokens, dtype=torch.bool, device="cuda")
        else:
            gone = torch.arange(tokens, device="cuda") % 4 == 1
        if kind == "ignored":
            y[gone] = 3
            gone = y == 3
            ignore = 3
        else:
            y[gone] = vocab if kind == "beyond" else -1 if kind != "last" else -(1 << 40)
        # what hidden holds at masked tokens does not matter
        x[gone] = float("nan")
        x[gone.nonzero()[::2, 0]] = float("inf")
        for reduction in ("mean", "sum", "none"):
            loss, gx, gw = head_check(x, table, y, reduction=reduction, ignore_id=ignore)
            assert bool((gx[gone] == 0).all())
            if kind == "all":
                assert bool((loss == 0).all()) and bool((gw == 0).all())


def test_head_targets_in_longer_rows_and_shifted_ids():
    hidden, table, targets = head_inputs(6 * 20, 300, 64, "bf16")
    long = torch.full((6, 33), 7, device="cuda")
    long[:, 5:25] = targets.view(6, 20)
    a = head_check(hidden.view(6, 20, 64), table, long[:, 5:25], reduction="none")
    b = head_check(hidden.view(6, 20, 64), table, (long[:, 5:25] + 1000).int(), reduction="none", first_id=1000)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    c = g.linear_cross_entropy(hidden, table, targets, reduction="none")
    assert torch.equal(c.view(6, 20), a[0])
    # hidden's rows apart, at odd addresses, transposed; the table too
    for x in (padded(hidden, 8), padded(hidden, 3), shifted(hidden), hidden.t().contiguous().t()):
        for w in (table, padded(table, 8), padded(table, 1), shifted(table)):
            assert torch.equal(g.linear_cross_entropy(x, w, targets, reduction="none"), c)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("grad", ["bf16", "fp16", "fp32"])
def test_head_gradient_types_and_buffers(grad, dtype):
    hidden, table, targets = head_inputs(70, 200, 64, dtype)
    for accumulate in (False, True):
        head_check(hidden, table, targets, grad=grad, accumulate=accumulate, up=3.0)
    lse, _ = g.head_stats(hidden, table, targets)
    buf = torch.full((72, 70), 4.0, dtype=DT[grad], device="cuda")
    one = torch.ones(1, device="cuda")
    gx, gw = g.head_grad(hidden, table, targets, lse, one, reduction="mean", grad_hidden=buf[1:-1, 2:66])
    assert gx.data_ptr() == buf[1:-1, 2:66].data_ptr() and gw is None
    for edge in (buf[0], buf[-1], buf[:, :2], buf[:, 66:]):
        assert bool((edge == 4.0).all())
    x = hidden.detach().requires_grad_()
    g.linear_cross_entropy(x, table, targets).backward()
    if grad == dtype:
        assert torch.equal(gx, x.grad)


@pytest.mark.parametrize("scale", [65536.0, 1e-6, 2.0 ** 60, 2.0 ** -60])
def test_head_loss_scales(scale):
    """fp16 gradients under a loss scale lose no probabilities; far scales in
    bf16, whose range has room."""
    hidden, table, targets = head_inputs(64, 3000, 64, "fp16" if 1e-7 < scale < 1e6 else "bf16")
    if scale == 65536.0:
        head_check(hidden, table, targets, reduction="mean", up=scale)
    else:
        head_check(hidden.bfloat16(), table.bfloat16(), targets, reduction="mean", up=scale)


@pytest.mark.parametrize("vocab", [300, 40000])
@pytest.mark.parametrize("tokens", [1, 20, 129, 256, 257])
def test_head_masked_tokens_of_a_table_with_nan(tokens, vocab):
    """Their loss and gradient are 0 and they add nothing, whatever the table and their rows hold."""
    hidden, table, targets = head_inputs(tokens, vocab, 40, "bf16")
    table[7, 3], table[250] = float("nan"), float("inf")
    hidden[::2] = float("nan")
    targets[::2] = -1
    for y in (targets, torch.full_like(targets, -1)):
        x, w = hidden.detach().requires_grad_(), table.detach().requires_grad_()
        loss = g.linear_cross_entropy(x, w, y, reduction="none")
        loss.backward(torch.ones_like(loss))
        masked = y < 0
        assert bool((loss[masked] == 0).all()) and bool((x.grad[masked] == 0).all())
        assert bool(loss[~masked].isnan().all()) and bool(x.grad[~masked].isnan().all())
        if bool(masked.all()):
            assert bool((w.grad == 0).all())
            assert float(g.linear_cross_entropy(x, w, y)) == 0.0


def test_head_scale_of_nothing():
    """All logits 0, whatever the products are."""
    hidden, table, targets = head_inputs(70, 301, 40, "bf16")
    targets[::9] = -1
    loss = head_check(hidden, table, targets, scale=0.0)[0]
    assert abs(loss.item() - math.log(301)) < 1e-5


def test_head_weights_of_very_different_size():
    hidden, table, targets = head_inputs(64, 300, 64, "bf16")
    x, w = hidden.detach().requires_grad_(), table.detach().requires_grad_()
    weights = torch.exp2(torch.arange(64, device="cuda").float() - 40)
    weights[5] = 0.0
    g.linear_cross_entropy(x, w, targets, reduction="none").backward(weights)
    unit = head_check(hidden, table, targets, reduction="sum")[1]
    # a row's gradient scales with its weight, a power of two
    assert torch.equal(x.grad[10:], unit[10:] * weights[10:, None])
    assert bool((x.grad[5] == 0).all())


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_head_of_what_is_no_number(value):
    hidden, table, targets = head_inputs(40, 300, 64, "bf16")
    hidden[7, 3] = value
    x, w = hidden.detach().requires_grad_(), table.detach().requires_grad_()
    loss = g.linear_cross_entropy(x, w, targets, reduction="none")
    assert not bool(torch.isfinite(loss[7])) and int((~torch.isfinite(loss)).sum()) == 1
    loss.sum().backward()
    assert not bool(torch.isfinite(w.grad).all())
    rows = torch.isfinite(x.grad).all(1)
    assert not bool(rows[7]) and int((~rows).sum()) == 1
    # a gradient that is none (an overflown loss scale) is not hidden either
    x, w = head_inputs(40, 300, 64, "bf16")[0].requires_grad_(), table.detach().requires_grad_()
    g.linear_cross_entropy(x, w, targets).backward(torch.tensor(value, device="cuda"))
    assert not bool(torch.isfinite(x.grad).any()) and not bool(torch.isfinite(w.grad).any())


def test_head_of_far_logits():
    # logits of +-20000: the maximum leaves every exp in range
    hidden, table, targets = head_inputs(50, 400, 64, "bf16", sigma=30.0, know=False)
    hidden *= 40
    head_check(hidden, table, targets, reduction="none")
    head_check(hidden, table, targets, reduction="none", scale=-1.0)
    head_check(hidden, table, targets, reduction="none", scale=0.0)


@pytest.mark.parametrize("tokens,vocab,dim", [(4100, 40_000, 64), (300_000, 700, 24)])
def test_head_in_pieces_of_the_vocabulary(tokens, vocab, dim):
    """More logits than a piece's workspace, against float64 by stretches of tokens."""
    hidden, table, targets = head_inputs(tokens, vocab, dim, "bf16")
    targets[5::7] = -1
    x, w = hidden.detach().requires_grad_(), table.detach().requires_grad_()
    gw = torch.zeros(vocab, dim, device="cuda")
    loss = g.linear_cross_entropy(x, w, targets, grad_weight=gw)
    loss.backward()
    total, dw, dw_err = 0.0, torch.zeros(vocab, dim, dtype=torch.float64, device="cuda"), None
    dw_err = torch.zeros_like(dw)
    kept = int((targets >= 0).sum())
    W = table.double()
    step = max(1, 40_000_000 // vocab)
    for a in range(0, tokens, step):
        y = targets[a:a + step]
        counts = y >= 0
        X, _, logits, lse, d, e = head64(hidden[a:a + step], table, y, 1.0, counts)
        at = y.clamp(min=0)
        idx = torch.arange(y.numel(), device="cuda")
        total += float(torch.where(counts, lse - logits[idx, at], torch.zeros_like(lse)).sum())
        p = torch.exp(logits - lse[:, None])
        z = p.clone()
        z[idx, at] -= 1.0
        z = torch.where(counts[:, None], z / kept, torch.zeros_like(z))
        z_err = torch.where(counts[:, None], p / kept * (d + e[:, None] + 2.0 ** -22), torch.zeros_like(z)) + \
            (2.0 ** -8 + 4 * U) * z.abs()
        want = z @ W
        err = z_err @ W.abs() + 2 * U * (vocab + 8) * (z.abs() @ W.abs()) + rounded(want, torch.bfloat16)
        assert_close(x.grad[a:a + step], want, err, "grad_hidden")
        dw += z.t() @ X
        dw_err += z_err.t() @ X.abs() + 2 * U * (tokens + 2) * (z.abs().t() @ X.abs())
    assert abs(float(loss.detach()) - total / kept) <= 1e-5 * abs(total / kept) + 1e-5
    assert_close(gw, dw, dw_err + rounded(dw, torch.float32), "grad_weight")


@pytest.mark.parametrize("tokens", [3, 300])
def test_head_offsets_beyond_32_bits(tokens):
    vocab, dim = 280000, 8192
    table = torch.empty(vocab, dim, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.02).requires_grad_()
    hidden = randn((tokens, dim), torch.bfloat16, 2).requires_grad_()
    targets = torch.arange(tokens, device="cuda") * 7 + (vocab - 7 * tokens)
    g.linear_cross_entropy(hidden, table, targets, reduction="none").sum().backward()
    own = torch.arange(tokens, device="cuda")
    X, parts = hidden.detach().double(), list(range(0, vocab, 10000))
    logits, d = [], []
    for a in parts:
        W = table.detach()[a:a + 10000].double()
        logits.append(X @ W.t())
        d.append(2 * U * (dim + 2) * (X.abs() @ W.abs().t()) + 2 * U * logits[-1].abs())
    logits, d = torch.cat(logits, 1), torch.cat(d, 1)
    lse = torch.logsumexp(logits, 1)
    e = d.amax(1) + (300 + 8) * U + 4 * U * (lse.abs() + logits.abs().amax(1))
    p = torch.exp(logits - lse[:, None])
    z = p.clone()
    z[own, targets] -= 1.0
    z_err = p * (d + e[:, None] + 2.0 ** -22) + 4 * U * z.abs() + H[torch.bfloat16][0] * z.abs() + 2.0 ** -38
    want, err = torch.zeros_like(X), torch.zeros_like(X)
    for a in parts:
        W = table.detach()[a:a + 10000].double()
        want += z[:, a:a + 10000] @ W
        err += z_err[:, a:a + 10000] @ W.abs() + 2 * U * (vocab + 8) * (z[:, a:a + 10000].abs() @ W.abs())
    assert_close(hidden.grad, want, err + rounded(want, torch.bfloat16), "grad_hidden")
    for rows in (slice(0, 500), slice(vocab - 2500, vocab)):
        want = z[:, rows].t() @ X
        err = z_err[:, rows].t() @ X.abs() + 2 * U * (tokens + 4) * (z[:, rows].abs().t() @ X.abs())
        assert_close(table.grad[rows], want, err + rounded(want, torch.bfloat16), "grad_weight")


def test_head_of_ranks_that_split_the_vocabulary():
    hidden, table, targets = head_inputs(90, 1000, 64, "bf16")
    targets[4::9] = -1
    counts = targets >= 0
    whole = hidden.detach().requires_grad_(), table.detach().requires_grad_()
    loss = g.linear_cross_entropy(*whole, targets, reduction="none")
    weights = randn((90,), torch.float32, 5)
    loss.backward(weights)
    ranges = [(0, 300), (300, 301), (301, 1000)]
    stats = [g.head_stats(hidden, table[a:b], targets, first_id=a, classes=1000) for a, b in ranges]
    for lse, logit in stats:
        assert bool((lse[~counts] == 0).all()) and bool((logit[~counts] == 0).all())
    lse = torch.logsumexp(torch.stack([s[0] for s in stats]).double(), 0)
    logit = torch.stack([s[1] for s in stats]).double().sum(0)
    got = torch.where(counts, lse - logit, torch.zeros_like(lse))
    # both sides are within the loss's own error of float64
    _, _, logits, _, d, e = head64(hidden, table, targets, 1.0, counts)
    assert bool(((got - loss.detach().double()).abs() <= 4 * e).all())
    lse = lse.float()
    parts = [g.head_grad(hidden, table[a:b], targets, lse, weights, first_id=a, classes=1000,
                         grad_weight=torch.zeros(b - a, 64, dtype=torch.bfloat16, device="cuda"),
                         grad_hidden=torch.zeros(90, 64, device="cuda")) for a, b in ranges]
    p = torch.exp(logits - torch.logsumexp(logits, 1, keepdim=True))
    z = p.clone()
    z[torch.arange(90, device="cuda"), targets.clamp(min=0)] -= 1
    wt = torch.where(counts, weights.double(), torch.zeros_like(weights.double()))[:, None]
    z, z_err = z * wt, (p * (d + 2 * e[:, None] + 2.0 ** -21) + (2.0 ** -8 + 4 * U) * z.abs()) * wt.abs() + 2.0 ** -38
    X = torch.where(counts[:, None], hidden.double(), torch.zeros_like(hidden.double()))
    want = z @ table.double()
    assert_close(sum(x for x, _ in parts), want, z_err @ table.double().abs() + 2 * U * 1010 * (z.abs() @ table.double().abs()) +
                 rounded(want, torch.float32) * 3, "grad_hidden")
    want = z.t() @ X
    assert_close(torch.cat([w for _, w in parts]), want,
                 z_err.t() @ X.abs() + 2 * U * 92 * (z.abs().t() @ X.abs()) + rounded(want, torch.bfloat16), "grad_weight")


def test_head_gradient_against_differences():
    hidden, table, targets = head_inputs(24, 100, 40, "bf16")
    targets[3] = -1
    x, w = hidden.detach().requires_grad_(), table.detach().requires_grad_()
    gw = torch.zeros(100, 40, device="cuda")
    g.linear_cross_entropy(x, w, targets, scale=0.7, grad_weight=gw).backward()
    counts = targets >= 0

    def loss(h, t):
        logits = 0.7 * h @ t.t()
        each = torch.logsumexp(logits, 1) - logits.gather(1, targets.clamp(min=0)[:, None])[:, 0]
        return (each * counts).sum() / counts.sum()

    X, W, step = hidden.double(), table.double(), 1e-4
    for seed in range(4):
        dx, dw = randn((24, 40), torch.float64, seed), randn((100, 40), torch.float64, seed + 10)
        near = (loss(X + step * dx, W) - loss(X - step * dx, W)) / (2 * step)
        # the gradient's own error: half a step of bf16 for its rounding, as much for z's
        allowed = float((2.0 ** -7 * x.grad.double().abs() * dx.abs()).sum()) + 1e-6
        assert abs(float((x.grad.double() * dx).sum() - near)) <= allowed
        near = (loss(X, W + step * dw) - loss(X, W - step * dw)) / (2 * step)
        y = targets.clamp(min=0)
        z = torch.softmax(0.7 * X @ W.t(), 1)
        z[torch.arange(24, device="cuda"), y] -= 1
        bound = 2.0 ** -8 * 0.7 * ((z * counts[:, None]).abs().t() @ X.abs()) / counts.sum()
        assert abs(float((gw.double() * dw).sum() - near)) <= float((bound * dw.abs()).sum()) + 1e-6


def test_head_empty():
    table = randn((10, 8), torch.bfloat16, 1).requires_grad_()
    x = torch.zeros(0, 8, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    y = torch.zeros(0, dtype=torch.int64, device="cuda")
    for reduction in ("mean", "sum", "none"):
        loss = g.linear_cross_entropy(x, table, y, reduction=reduction)
        assert loss.shape == (() if reduction != "none" else (0,)) and bool((loss == 0).all())
        into = torch.full((10, 8), 3.0, device="cuda")
        loss = g.linear_cross_entropy(x, table, y, reduction=reduction, grad_weight=into, accumulate=True)
        loss.backward(torch.ones_like(loss))
        assert bool((into == 3.0).all())
        loss = g.linear_cross_entropy(x, table, y, reduction=reduction, grad_weight=into)
        loss.backward(torch.ones_like(loss))
        assert bool((into == 0.0).all())
    # no columns: every logit is 0
    x = torch.zeros(3, 0, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    w = torch.zeros(10, 0, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    loss = g.linear_cross_entropy(x, w, torch.tensor([1, 2, -1], device="cuda"), reduction="none")
    assert_close(loss.detach(), torch.tensor([math.log(10)] * 2 + [0.0], dtype=torch.float64, device="cuda"),
                 torch.full((3,), 1e-6, device="cuda"))
    loss.sum().backward()
    assert x.grad.shape == (3, 0) and w.grad.shape == (10, 0)
    # no classes: every token is masked
    x = torch.ones(3, 8, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    w = torch.zeros(0, 8, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    loss = g.linear_cross_entropy(x, w, torch.tensor([1, 2, -1], device="cuda"))
    loss.backward()
    assert float(loss.detach()) == 0.0 and bool((x.grad == 0).all()) and w.grad.shape == (0, 8)


def test_head_without_tokens_over_memory_that_held_nan():
    """What a workspace held before does not reach the gradients of no tokens."""
    for _ in range(3):
        junk = [torch.full((1 << k,), float("nan"), device="cuda") for k in range(6, 16)]
        del junk
        table = randn((10, 8), torch.bfloat16, 1).requires_grad_()
        x = torch.zeros(0, 8, dtype=torch.bfloat16, device="cuda", requires_grad=True)
        g.linear_cross_entropy(x, table, torch.zeros(0, dtype=torch.int64, device="cuda")).backward()
        assert bool((table.grad == 0).all())


def test_transposed_inputs_on_a_stream():
    x, w = randn((64, 600), torch.bfloat16, 1), randn((200, 600), torch.bfloat16, 2)
    want = g.linear8(x, w)
    s = torch.cuda.Stream()
    for _ in range(3):
        turned = x.t().contiguous().t()
        s.wait_stream(torch.cuda.current_stream())
        got = g.linear8(turned, w, stream=s)
        s.synchronize()
        assert torch.equal(got, want)


def test_rows_that_are_one_row_or_overlap():
    """Expanded inputs and gradients, and windows of one buffer, are what their copies are."""
    w, table = randn((72, 48), torch.bfloat16, 1), randn((200, 48), torch.bfloat16, 2)
    row, buf = randn((1, 48), torch.bfloat16, 3), randn((48 + 29 * 8,), torch.bfloat16, 4)
    targets = torch.arange(30, device="cuda")
    for x in (row.expand(30, 48), buf.as_strided((30, 48), (8, 1)), row[None].expand(5, 6, 48)):
        got = []
        for rows in (x, x.contiguous()):
            a, v = rows.detach().requires_grad_(), w.detach().requires_grad_()
            t = table.detach().requires_grad_()
            y = g.linear8(a, v)
            y.reshape(30, 72).sum(0).backward(w[:, 0])
            up = g.gate8(rows.detach().requires_grad_(), a)
            up.reshape(30, 48).sum(0).backward(row[0])
            g.linear_cross_entropy(a, t, targets.view(rows.shape[:-1]), reduction="none").sum().backward()
            got.append((y.detach(), up.detach(), a.grad, v.grad, t.grad, g.act8_pack(rows).unpack()))
        for one, other in zip(*got):
            assert torch.equal(one, other)


def test_more_tokens_than_a_block_holds_at_once():
    hidden, table, targets = head_inputs(40001, 60, 24, "bf16")
    targets[3::5] = -1
    targets[17000:18500] = -1
    head_check(hidden, table, targets, reduction="none")
    targets[:-1] = -1
    head_check(hidden, table, targets)


def test_head_gradients_that_are_not_wanted():
    hidden, table, targets = head_inputs(50, 300, 64, "bf16")
    both = hidden.detach().requires_grad_(), table.detach().requires_grad_()
    g.linear_cross_entropy(*both, targets).backward()
    x = hidden.detach().requires_grad_()
    into = torch.full((300, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    g.linear_cross_entropy(x, table, targets, grad_weight=into).backward()
    assert torch.equal(x.grad, both[0].grad) and bool((into == 9.0).all())
    w = table.detach().requires_grad_()
    g.linear_cross_entropy(hidden, w, targets).backward()
    assert torch.equal(w.grad, both[1].grad)


# ---- the ways calls are made ----------------------------------------------------------------


def test_the_same_bits_every_time_on_any_stream():
    hidden, table, targets = head_inputs(700, 5000, 96, "bf16")
    w = randn((176, 96), torch.bfloat16, 5)
    first = None
    for k in range(4):
        s = torch.cuda.Stream() if k % 2 else torch.cuda.current_stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            x, t, v = hidden.detach().requires_grad_(), table.detach().requires_grad_(), w.detach().requires_grad_()
            y = g.gate8(g.linear8(x, v))
            y.float().square().mean().backward()
            loss = g.linear_cross_entropy(x, t, targets)
            loss.backward()
            got = [y.detach(), loss.detach(), x.grad, t.grad, v.grad]
        s.synchronize()
        if first is None:
            first = got
        for a, b in zip(got, first):
            assert torch.equal(a, b)


def test_two_calls_at_once_on_two_streams():
    a, b = head_inputs(900, 3000, 128, "bf16", 1), head_inputs(900, 3000, 128, "bf16", 9)
    alone = [g.linear_cross_entropy(*x, reduction="none") for x in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [g.linear_cross_entropy(*x, reduction="none", stream=s) for x, s in zip((a, b), streams)]
        torch.cuda.synchronize()
        assert torch.equal(got[0], alone[0]) and torch.equal(got[1], alone[1])


def test_a_captured_step_replays():
    """Forward and backward of all operators in one graph, with new inputs between
    replays, eager work between them, against eager calls."""
    table = randn((500, 64), torch.bfloat16, 1, 0.1)
    w1, w2 = randn((2 * 96, 64), torch.bfloat16, 2, 0.1), randn((64, 96), torch.bfloat16, 3, 0.1)
    targets = torch.randint(0, 500, (4, 33), device="cuda")
    leaves = [t.detach().requires_grad_() for t in (table, w1, w2)]
    into = [torch.zeros_like(t) for t in (table, w1, w2)]
    static = targets.clone()

    def run():
        # the head's backward runs first and writes the table's gradient, the lookup's adds to it
        h = g.embedding(leaves[0], static, grad_weight=into[0], accumulate=True)
        a = g.linear8(h, leaves[1], grad_weight=into[1])
        h = h + g.linear8(g.gate8(a[..., :96], a[..., 96:]), leaves[2], grad_weight=into[2])
        loss = g.linear_cross_entropy(h[:, :-1], leaves[0], static[:, 1:], grad_weight=into[0])
        loss.backward()
        return loss.detach()

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
        fresh = torch.randint(0, 500, (4, 33), device="cuda")
        fresh[1, 20:] = -1
        if k == 2:
            fresh[:] = -1
        static.copy_(fresh)
        for t in into:
            t.fill_(float("nan"))
        graph.replay()
        got = [captured.clone(), *(t.clone() for t in into)]
        torch.cuda.synchronize()
        want = run()
        for a, b in zip(got, [want, *into]):
            assert torch.equal(a, b), k
        assert torch.isfinite(got[0])


def test_a_training_step_through_all_operators():
    """The operators around the step and of the model as one training step: tied
    table, gradients into a Session's flat gradient, clip, step; against float64."""
    V, D, F, B, L = 400, 64, 96, 6, 40
    sizes = [V * D, 2 * F * D, D * F]
    n = sum(sizes)
    clipped = g.GradResult()
    sess = g.Session(n, ring_bytes=1 << 20, init_scale=256.0, found_inf=clipped.found_inf, grad_norm=False)
    try:
        with torch.cuda.stream(sess.compute):
            sess.master.copy_(randn((n,), torch.float32, 1, 0.1))
            sess.weight.copy_(sess.master)
            parts = torch.split(sess.weight, sizes)
            grads = torch.split(sess.grad, sizes)
            shapes = [(V, D), (2 * F, D), (D, F)]
            table, w1, w2 = (p.view(s).detach().requires_grad_() for p, s in zip(parts, shapes))
            gt, g1, g2 = (p.view(s) for p, s in zip(grads, shapes))
            clip = g.GradList([gt, g1, g2], stream=sess.compute)
            ids = torch.randint(0, V, (B, L), device="cuda")
            ids[2, 30:] = -1
            before = [p.double().view(s).clone() for p, s in zip(parts, shapes)]
            sess.backward_begin()
            h = g.embedding(table, ids, grad_weight=gt, accumulate=True)
            a = g.linear8(h, w1, grad_weight=g1)
            h2 = h + g.linear8(g.gate8(a[..., :F], a[..., F:]), w2, grad_weight=g2)
            loss = g.linear_cross_entropy(h2[:, :-1], table, ids[:, 1:], grad_weight=gt)
            (loss * 256.0).backward()
            raw = [x.double().clone() / 256.0 for x in (gt, g1, g2)]
            r = clip.clip(0.05, scale=sess, result=clipped)
            sess.step(1e-3)
            after = sess.weight.clone()
        torch.cuda.synchronize()
    finally:
        sess.close()
    T, W1, W2 = (t.requires_grad_() for t in before)
    there = (ids >= 0)[..., None]
    H0 = T[ids.clamp(min=0)] * there
    A = H0 @ W1.t()
    H2 = H0 + (torch.nn.functional.silu(A[..., :F]) * A[..., F:]) @ W2.t()
    logits = H2[:, :-1] @ T.t()
    want = ids[:, 1:]
    each = torch.logsumexp(logits, -1) - logits.gather(-1, want.clamp(min=0)[..., None])[..., 0]
    kept = want >= 0
    total = (each * kept).sum() / kept.sum()
    total.backward()
    # the 16-bit activations between the layers make most of the difference: a few
    # roundings of 2^-9 (mean) each, and 8 bits' 2^-8 of a block's largest
    assert abs(float(loss) - float(total)) <= 2.0 ** -7 * float(total)
    for got, t in zip(raw, (T, W1, W2)):
        assert float((got - t.grad).norm()) <= 0.03 * float(t.grad.norm())
    norm = math.sqrt(sum(float(x.square().sum()) for x in raw))
    assert abs(float(r.norm) - norm) <= 1e-4 * norm and float(r.found_inf) == 0.0
    assert not torch.equal(after, torch.cat([b.detach().reshape(-1) for b in before]).bfloat16())


def test_refusals():
    x, w = randn((4, 8), torch.bfloat16, 1), randn((6, 8), torch.bfloat16, 2)
    y = torch.zeros(4, dtype=torch.int64, device="cuda")
    s = torch.cuda.Stream()
    for call in (lambda: g.linear_cross_entropy(x, w, y, reduction="max"),
                 lambda: g.linear_cross_entropy(x, w, y[:3]),
                 lambda: g.linear_cross_entropy(x, w[:, :7], y),
                 lambda: g.linear_cross_entropy(x, w, y.float()),
                 lambda: g.linear_cross_entropy(x, w[0], y),
                 lambda: g.linear_cross_entropy(x.clone().requires_grad_(), w, y, stream=s),
                 lambda: g.linear_cross_entropy(x, w.clone().requires_grad_(), y, accumulate=True),
                 lambda: g.linear_cross_entropy(x, w.clone().requires_grad_(), y, grad_weight=w[:3]),
                 lambda: g.linear_cross_entropy(x, w.clone().requires_grad_(), y, grad_weight=w.t().contiguous().t()),
                 lambda: g.linear_cross_entropy(x, w.clone().requires_grad_(), y,
                                                grad_weight=w.clone().requires_grad_()),
                 lambda: g.linear_cross_entropy(x.cpu(), w, y), lambda: g.linear_cross_entropy(x, w, y.cpu()),
                 lambda: g.head_grad(x, w, y, torch.zeros(3, device="cuda"), torch.zeros(4, device="cuda")),
                 lambda: g.head_grad(x, w, y, torch.zeros(4, device="cuda"), torch.zeros(1, device="cuda")),
                 lambda: g.head_grad(x, w, y, torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"), accumulate=True),
                 lambda: g.linear8(x, w[:, :4]), lambda: g.linear8(x, w[0]), lambda: g.linear8(x.cpu(), w),
                 lambda: g.linear8(x, w.clone().requires_grad_(), stream=s),
                 lambda: g.linear8_grad_weight(x, g.act8_pack(x), w),
                 lambda: g.linear8_grad_weight(x[:2], g.act8_pack(x), torch.zeros(8, 8, device="cuda")),
                 lambda: g.gate8(x, kind="relu"), lambda: g.gate8(x, x[:2]), lambda: g.gate8(x, x.float()),
                 lambda: g.gate8(x.clone().requires_grad_(), stream=s), lambda: g.gate8(x[0, 0]),
                 lambda: g.act8_pack(x[0, 0]), lambda: g.act8_pack(x.int()), lambda: g.act8_pack(x, out=g.act8_pack(x[:2])),
                 lambda: g.act8_pack(x).unpack(out=torch.zeros(3, 8, device="cuda")),
                 lambda: g.Act8((3, 4), torch.float64)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: g.linear_cross_entropy(x.float(), w.float(), y), lambda: g.linear_cross_entropy(x.half(), w, y),
                 lambda: g.linear8(x.float(), w.float()), lambda: g.linear8(x, w.half()),
                 lambda: g.head_stats(x, w, y, first_id=3, classes=8)):
        with pytest.raises(g.GockptError):
            call()
    import torch.autograd.forward_ad as fwAD
    with fwAD.dual_level():
        d = fwAD.make_dual(x, torch.ones_like(x))
        for call in (lambda: g.linear_cross_entropy(d, w, y), lambda: g.linear8(d, w), lambda: g.gate8(d)):
            with pytest.raises(NotImplementedError):
                call()
