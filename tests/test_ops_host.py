"""The operators of include/gockpt_ops.h on the CPU: structs and exports of
the binding against the header, workspace sizes, and the refusals of the C
entry points (all of them come before any device call)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

import paper_2511_07035_amd as g
from paper_2511_07035_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gockpt_ops.h")
P = 1 << 20  # stands for a device address, never read here
BF16, FP16, FP32 = 0, 1, 2

FIELDS = {
    "gockpt_grad_tensor": (ops.GRAD_TENSOR, ["data", "dst", "rows", "cols", "stride", "dtype", "dst_dtype"]),
    "gockpt_grad_result": (ops.GRAD_RESULT, ["sumsq", "norm", "found_inf", "coef", "reserved_"]),
    "gockpt_token_ids": (ops.TOKEN_IDS, ["ids", "batch", "length", "stride", "first_id", "bits", "reserved_"]),
    "gockpt_matrix": (ops.MATRIX, ["data", "rows", "cols", "stride", "dtype", "reserved_"]),
}


def test_packed_structs_match_the_header(tmp_path):
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no C compiler")
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    assert set(re.findall(r"\}\s*(gockpt_\w+)\s*;", text)) == set(FIELDS)
    lines, expect = [], []
    for name, (fmt, fields) in FIELDS.items():
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        expect.append(fmt.size)
        at = 0
        codes = re.findall(r"(\d*)([a-zA-Z])", fmt.format)
        flat = []
        for n, c in codes:
            flat += [c] * int(n or 1) if not n else [n + c]
        assert len(flat) == len(fields)
        for c, f in zip(flat, fields):
            lines.append(f'  printf("%zu\\n", offsetof({name}, {f}));')
            expect.append(at)
            at += ops.struct.calcsize("<" + c)
    src = tmp_path / "layout.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"gockpt_ops.h\"\nint main(void) {\n"
                   + "\n".join(lines) + "\n  return 0;\n}\n")
    exe = tmp_path / "layout"
    r = subprocess.run([cc, "-std=c99", "-Wall", "-Werror", f"-I{ROOT}/include", str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in got] == expect


def test_library_exports_every_declared_function():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(gockpt_[a-z_0-9]+)\s*\(", text)))
    assert "gockpt_grads_clip" in names and "gockpt_embedding_grad" in names
    L = g.lib()
    assert [n for n in names if not hasattr(L, n)] == []


def _error():
    return g.lib().gockpt_last_error(None).decode()


def _bytes(*tensors):
    n = ctypes.c_size_t(99)
    rc = ops._lib().gockpt_grads_bytes(b"".join(ops.GRAD_TENSOR.pack(*t) for t in tensors), len(tensors),
                                       ctypes.byref(n))
    return rc, n.value


@pytest.mark.parametrize("tensor,said", [
    ((P, 0, 1, 8, 8, 3, 0), "dtype 3"),
    ((P, P, 1, 8, 8, BF16, -1), "dst_dtype -1"),
    ((P, 0, -1, 8, 8, BF16, 0), "-1 x 8"),
    ((P, 0, 2, -8, 8, BF16, 0), "2 x -8"),
    ((P, 0, 1 << 40, 1 << 40, 1 << 40, BF16, 0), "elements"),
    ((P, 0, 2, 8, 7, BF16, 0), "stride 7"),
    ((P, 0, 2, 8, 0, BF16, 0), "stride 0"),
    ((0, 0, 1, 8, 8, BF16, 0), "null"),
    ((P + 1, 0, 1, 8, 8, BF16, 0), "aligned"),
    ((P + 2, 0, 1, 8, 8, FP32, 0), "aligned"),
    ((P, P + 2, 1, 8, 8, BF16, FP32), "dst is not aligned"),
    ((P, P, 1, 8, 8, FP32, BF16), "another type"),
    ((P, P, 2, 8, 9, BF16, BF16), "another type or layout"),
])
def test_tensor_refusals(tensor, said):
    good = (P, 0, 1, 8, 8, BF16, 0)
    rc, n = _bytes(good, tensor)
    assert rc == g.GOCKPT_EINVAL and n == 0
    assert "tensor 1" in _error() and said in _error(), _error()


def test_list_sizes_and_refusals():
    L = ops._lib()
    rc, none = _bytes()
    assert rc == 0 and none % 256 == 0
    # 16 KiB a table entry of 48 bytes; rows apart share entries while they fit
    for t, entries in (((P, 0, 1, 8192, 8192, BF16, 0), 1), ((P, 0, 1, 8193, 8193, BF16, 0), 2),
                       ((P, 0, 1, 4097, 4097, FP32, 0), 2), ((P, 0, 300, 10, 10, BF16, 0), 1),
                       ((P, 0, 513, 10, 11, BF16, 0), 2), ((P, 0, 3, 8193, 8200, FP16, 0), 6),
                       ((P, 0, 7, 4097, 5000, BF16, 0), 7), ((P, 0, 0, 5, 5, BF16, 0), 0),
                       ((P, 0, 5, 0, 5, BF16, 0), 0)):
        rc, n = _bytes(t)
        assert rc == 0 and n == (none + 48 * entries + 255) // 256 * 256, (t, n, none)
    n = ctypes.c_size_t()
    assert L.gockpt_grads_bytes(None, 1, ctypes.byref(n)) == g.GOCKPT_EINVAL
    assert L.gockpt_grads_bytes(b"", -1, ctypes.byref(n)) == g.GOCKPT_EINVAL
    assert L.gockpt_grads_bytes(b"", 0, None) == g.GOCKPT_EINVAL
    h = ctypes.c_void_p(7)
    t = ops.GRAD_TENSOR.pack(P, 0, 1, 8, 8, BF16, 0)
    assert L.gockpt_grads_create(t, 1, None, 1 << 20, None, ctypes.byref(h)) == g.GOCKPT_EINVAL and not h.value
    assert L.gockpt_grads_create(t, 1, P + 16, 1 << 20, None, ctypes.byref(h)) == g.GOCKPT_EINVAL
    assert L.gockpt_grads_create(t, 1, P, 64, None, ctypes.byref(h)) == g.GOCKPT_ENOMEM
    assert L.gockpt_grads_create(t, 1, P, 1 << 20, None, None) == g.GOCKPT_EINVAL
    assert L.gockpt_grads_destroy(None) == 0
    for f in (L.gockpt_grads_norm, L.gockpt_grads_clip):
        assert f(None, None, 1.0, P, None) == g.GOCKPT_EINVAL
    assert L.gockpt_grads_scale(None, P, None) == g.GOCKPT_EINVAL
    for scale, most, result in ((None, 1.0, None), (None, 1.0, P + 4), (P + 2, 1.0, P), (None, -1.0, P),
                                (None, float("nan"), P)):
        assert L.gockpt_grads_result(result, scale, most, None) == g.GOCKPT_EINVAL
    assert L.gockpt_scale_ptr(None, ctypes.byref(h)) == g.GOCKPT_EINVAL
    assert L.gockpt_scale_ptr(None, None) == g.GOCKPT_EINVAL


MATRIX = dict(table=(P, 100, 64, 64, BF16, 0), out=(P, 6, 64, 64, BF16, 0))
TOKENS = (P, 2, 3, 3, 0, 64, 0)


@pytest.mark.parametrize("change,said", [
    (dict(table=(P, 100, 64, 64, 5, 0)), "dtype 5"),
    (dict(table=(P, -1, 64, 64, BF16, 0)), "-1 x 64"),
    (dict(table=(P, 100, 1 << 25, 1 << 25, BF16, 0)), "x 33554432"),
    (dict(table=(P, 100, 64, 63, BF16, 0)), "stride 63"),
    (dict(table=(0, 100, 64, 64, BF16, 0)), "null"),
    (dict(table=(P + 1, 100, 64, 64, BF16, 0)), "aligned"),
    (dict(out=(P, 7, 64, 64, BF16, 0)), "6 tokens, 7 rows"),
    (dict(out=(P, 6, 65, 65, BF16, 0)), "columns"),
    (dict(out=(P + 2, 6, 64, 64, FP32, 0)), "aligned"),
    (dict(tokens=(P, -2, -3, 3, 0, 64, 0)), "tokens"),
    (dict(tokens=(P, 1 << 20, 1 << 20, 1 << 20, 0, 64, 0)), "tokens"),
    (dict(tokens=(P, 2, 3, 2, 0, 64, 0)), "ids stride 2"),
    (dict(tokens=(P, 2, 3, 3, 0, 16, 0)), "16 bits"),
    (dict(tokens=(0, 2, 3, 3, 0, 64, 0)), "null"),
    (dict(tokens=(P + 4, 2, 3, 3, 0, 64, 0)), "not aligned"),
])
def test_embedding_refusals(change, said):
    L = ops._lib()
    case = dict(MATRIX, tokens=TOKENS, **{}) | change
    table, out = ops.MATRIX.pack(*case["table"]), ops.MATRIX.pack(*case["out"])
    tokens = ops.TOKEN_IDS.pack(*case["tokens"])
    assert L.gockpt_embedding(table, tokens, 1.0, out, None) == g.GOCKPT_EINVAL
    assert said in _error(), _error()
    # the gradient reads `out` and writes `table`
    assert L.gockpt_embedding_grad(out, tokens, ops.NO_PADDING, 1.0, 0, table, None, 0, None) == g.GOCKPT_EINVAL
    assert said in _error(), _error()


def test_embedding_grad_sizes_and_refusals():
    L = ops._lib()
    size = g.gockpt_embedding_grad_bytes
    assert size(0, 100, 64) == 0 and size(16, 50304, 2048) == 0
    big = size(16384, 50304, 2048)
    assert big > 16384 * 8 and big % 256 == 0
    with pytest.raises(g.GockptError):
        size(16, (1 << 22) + 1, 8)
    with pytest.raises(g.GockptError):
        size(-1, 10, 8)
    grad = ops.MATRIX.pack(P, 16384, 64, 64, BF16, 0)
    tokens = ops.TOKEN_IDS.pack(P, 1, 16384, 16384, 0, 32, 0)
    table = ops.MATRIX.pack(P, 100, 64, 64, BF16, 0)
    need = size(16384, 100, 64)
    call = L.gockpt_embedding_grad
    assert call(grad, tokens, 0, 1.0, 0, table, None, 0, None) == g.GOCKPT_EINVAL
    assert call(grad, tokens, 0, 1.0, 0, table, P + 128, need, None) == g.GOCKPT_EINVAL
    assert call(grad, tokens, 0, 1.0, 0, table, P, need - 1, None) == g.GOCKPT_ENOMEM
    assert call(grad, tokens, 0, 1.0, 0, ops.MATRIX.pack(P, (1 << 22) + 1, 64, 64, BF16, 0), P, need, None) == \
        g.GOCKPT_EINVAL
    for args in ((None, tokens, table), (grad, None, table), (grad, tokens, None)):
        assert call(args[0], args[1], 0, 1.0, 0, args[2], P, need, None) == g.GOCKPT_EINVAL
        assert L.gockpt_embedding(args[2], args[1], 1.0, args[0], None) == g.GOCKPT_EINVAL
    # nothing to do: no launch, so no device either
    empty = ops.MATRIX.pack(0, 0, 64, 64, BF16, 0)
    no_tokens = ops.TOKEN_IDS.pack(0, 0, 16, 16, 0, 64, 0)
    assert L.gockpt_embedding(table, no_tokens, 1.0, empty, None) == 0
    assert call(empty, no_tokens, 0, 1.0, 1, table, None, 0, None) == 0
    assert call(ops.MATRIX.pack(P, 16384, 0, 0, BF16, 0), tokens, 0, 1.0, 0, ops.MATRIX.pack(P, 100, 0, 0, BF16, 0), None, 0,
                None) == 0


@pytest.mark.parametrize("shape,stride,want", [
    ((4, 5), (5, 1), (1, 20, 20)), ((4, 5), (8, 1), (4, 5, 8)), ((7,), (1,), (1, 7, 7)), ((7,), (3,), (7, 1, 3)),
    ((), (), (1, 1, 1)), ((1, 1), (9, 9), (1, 1, 1)), ((3, 0), (1, 1), (0, 0, 0)),
    ((2, 3, 4), (12, 4, 1), (1, 24, 24)), ((2, 3, 4), (24, 8, 1), (6, 4, 8)), ((2, 3, 4), (100, 4, 1), (2, 12, 100)),
    ((2, 3, 4), (100, 8, 1), None), ((4, 5), (1, 4), None), ((4, 5), (0, 1), None), ((4, 5), (3, 1), None),
    ((5, 1, 4), (4, 77, 1), (1, 20, 20)),
])
def test_rows_of_strided_tensors(shape, stride, want):
    assert ops._rows(shape, stride) == want


def test_tensors_off_the_gpu_are_refused():
    import torch
    t = torch.zeros(8)
    with pytest.raises(ValueError):
        g.GradList([t])
    with pytest.raises(ValueError):
        g.embedding(torch.zeros(4, 8), torch.zeros(2, dtype=torch.int64), out=torch.zeros(2, 8))
    with pytest.raises(ValueError):
        g.embedding_grad(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64), torch.zeros(4, 8))


class _Stream:
    """Of a fake device: remembers what it has waited for."""

    def __init__(self, number):
        self.cuda_stream, self.waited = number, []

    def wait_stream(self, other):
        self.waited.append(other)


def test_a_list_orders_its_calls_across_streams(monkeypatch):
    import torch
    a, b, c = _Stream(1), _Stream(2), _Stream(3)
    captured = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(ops, "_capturing", lambda s: s in captured, raising=False)

    class Memory:
        recorded = []

        def record_stream(self, stream):
            self.recorded.append(stream)

    gl = ops.GradList.__new__(ops.GradList)
    gl.handle, gl.device, gl.last, gl.at, gl.streams = 7, 0, a, 1, {1}
    gl.workspace, gl.tensors, gl.out, gl.result = Memory(), [Memory()], [None], ops.GradResult("cpu")
    gl.result.buffer = Memory()
    assert [gl._on(s) for s in (a, b, b, c, a)] == [1, 2, 2, 3, 1]
    assert a.waited == [c] and b.waited == [a] and c.waited == [b]
    assert Memory.recorded == [b] * 3 + [c] * 3  # once for each stream but the list's own
    # a call that a graph records runs later: nothing to wait for, and nothing ran
    captured.append(b)
    assert gl._on(b) == 2 and b.waited == [a]
    assert gl._on(c) == 3 and c.waited == [b, a]
    gl.handle = None


def test_a_result_off_the_lists_gpu_is_refused(monkeypatch):
    import torch

    class Calls:
        def __getattr__(self, name):
            return lambda *a: 0

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(ops, "_stream", lambda stream, device: 0)
    monkeypatch.setattr(ops, "_lib", lambda: Calls())
    monkeypatch.setattr(ops.GradList, "__del__", lambda self: None)
    gl = ops.GradList.__new__(ops.GradList)
    gl.handle, gl.device, gl.at, gl.result = 7, 0, 0, None
    off = g.GradResult("cpu")
    for call in (gl.norm, lambda result: gl.clip(1.0, result=result), gl.scale):
        with pytest.raises(ValueError):
            call(result=off)
    gl.handle = None


def test_a_sessions_scale_is_waited_for_on_other_streams(monkeypatch):
    import torch
    own, other, captured = _Stream(1), _Stream(2), []
    own.device_index = 0
    monkeypatch.setattr(ops, "_capturing", lambda s: s in captured)
    monkeypatch.setattr(ops, "gockpt_scale_ptr", lambda ctx: ctx + 1)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: other)

    class Sess:
        ctx, compute = 41, own

    assert ops._scale_ptr(Sess, 0, own, 1) == 42 and own.waited == []
    assert ops._scale_ptr(Sess, 0, other, 2) == 42 and other.waited == [own]
    assert ops._scale_ptr(Sess, 0, None, 2) == 42 and other.waited == [own, own]  # the current one
    captured.append(other)
    assert ops._scale_ptr(Sess, 0, other, 2) == 42 and other.waited == [own, own]
    with pytest.raises(ValueError):
        ops._scale_ptr(Sess, 1, other, 2)


def test_a_star_import_needs_no_torch():
    import sys
    code = ("import sys; sys.modules['torch'] = None\nfrom paper_2511_07035_amd import *\n"
            "print(gockpt_workspace_bytes(1000) > 0, Session.__name__)")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.stdout.split() == ["True", "Session"], r.stderr


@pytest.mark.parametrize("scale", [2.0, 65536, "1"])
def test_a_scale_of_another_kind_is_refused(scale):
    with pytest.raises(ValueError, match="scale"):
        ops._scale_ptr(scale, 0, None, 0)
