"""The operators of include/gockpt_model.h on the CPU: structs and exports of
the binding against the header, workspace sizes, and the refusals of the C entry
points (all of them come before any device call)."""
import ctypes
import os
import re
import shutil
import struct
import subprocess

import pytest

import paper_2511_07035_amd as g
from paper_2511_07035_amd import model, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gockpt_model.h")
P = 1 << 20  # stands for a device address, never read here
BF16, FP16, FP32 = 0, 1, 2
NONE = ops.NO_PADDING


def test_packed_structs_and_constants_match_the_header(tmp_path):
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no C compiler")
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    assert set(re.findall(r"\}\s*(gockpt_\w+)\s*;", text)) == {"gockpt_head", "gockpt_act8"}
    at = 2 * ops.MATRIX.size + ops.TOKEN_IDS.size
    want = {"sizeof(gockpt_head)": model.HEAD_SIZE, "offsetof(gockpt_head, table)": ops.MATRIX.size,
            "offsetof(gockpt_head, targets)": 2 * ops.MATRIX.size, "offsetof(gockpt_head, ignore_id)": at,
            "offsetof(gockpt_head, classes)": at + 8, "offsetof(gockpt_head, scale)": at + 16,
            "sizeof(gockpt_act8)": model.ACT8.size, "offsetof(gockpt_act8, scales)": 8,
            "offsetof(gockpt_act8, rows)": 16, "offsetof(gockpt_act8, cols)": 24}
    for name in re.findall(r"#define (GOCKPT_\w+) \d+", text):
        want[f"(size_t){name}"] = getattr(g, name)
    src = tmp_path / "layout.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"gockpt_model.h\"\nint main(void) {\n"
                   + "".join(f'  printf("%zu\\n", {e});\n' for e in want) + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    r = subprocess.run([cc, "-std=c99", "-Wall", "-Werror", f"-I{ROOT}/include", str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    assert dict(zip(want, map(int, got))) == want


def test_library_exports_every_declared_function():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(gockpt_[a-z_0-9]+)\s*\(", text)))
    assert len(names) == 12
    L = model._lib()
    for n in names:
        assert getattr(L, n).argtypes is not None, n


def test_the_package_offers_them():
    for n in ("linear_cross_entropy", "head_stats", "head_grad", "Act8", "act8_pack", "linear8", "linear8_grad_weight",
              "gate8"):
        assert getattr(g, n) is getattr(model, n)


def said():
    return g.lib().gockpt_last_error(None).decode()


def M(rows, cols, stride=None, dtype=BF16, data=P):
    return ops.MATRIX.pack(data, rows, cols, cols if stride is None else stride, dtype, 0)


def head(hidden=None, table=None, ids=(P, 2, 3, 3, 0, 64, 0), ignore=NONE, classes=0, scale=1.0):
    return (hidden or M(6, 64)) + (table or M(100, 64)) + ops.TOKEN_IDS.pack(*ids) + \
        model.HEAD_END.pack(ignore, classes, scale, 0)


def size(name, *args):
    n = ctypes.c_size_t(99)
    rc = getattr(model._lib(), name)(*args, ctypes.byref(n))
    return rc, n.value


@pytest.mark.parametrize("change,text", [
    (dict(hidden=M(6, 64, dtype=FP32)), "hidden dtype 2"),
    (dict(table=M(100, 64, dtype=5)), "table dtype 5"),
    (dict(table=M(100, 64, dtype=FP16)), "hidden of dtype 0, table of 1"),
    (dict(table=M(100, 65)), "hidden of 64 columns, table of 65"),
    (dict(hidden=M(-1, 64)), "-1 x 64"),
    (dict(hidden=M(6, 64, 63)), "stride 63"),
    (dict(hidden=M(6, 64, data=0)), "null"),
    (dict(hidden=M(6, 64, data=P + 1)), "aligned"),
    (dict(table=M(1 << 31, 64)), "2147483648 x 64"),
    (dict(table=M(100, 1 << 23), hidden=M(6, 1 << 23)), "x 8388608"),
    (dict(hidden=M(7, 64)), "6 targets, 7 rows"),
    (dict(ids=(P, -2, -3, 3, 0, 64, 0)), "targets"),
    (dict(ids=(P, 2, 3, 2, 0, 64, 0)), "targets stride 2"),
    (dict(ids=(P, 2, 3, 3, 0, 16, 0)), "16 bits"),
    (dict(ids=(0, 2, 3, 3, 0, 64, 0)), "null"),
    (dict(ids=(P + 4, 2, 3, 3, 0, 64, 0)), "not aligned"),
    (dict(ids=(P, 2, 3, 3, (1 << 63) - 5, 64, 0)), "first_id"),
    (dict(classes=-1), "classes"),
    (dict(classes=99), "0 to 100 of 99 classes"),
    (dict(classes=200, ids=(P, 2, 3, 3, 101, 64, 0)), "101 to 201 of 200 classes"),
    (dict(classes=200, ids=(P, 2, 3, 3, -1, 64, 0)), "-1 to 99 of 200 classes"),
])
def test_head_refusals(change, text):
    L, h = model._lib(), head(**change)
    for rc in (size("gockpt_head_loss_bytes", h)[0], size("gockpt_head_grad_bytes", h, None, None)[0],
               L.gockpt_head_loss(h, 0, P, P, P, P, 1 << 40, None),
               L.gockpt_head_grad(h, P, 0, P, M(6, 64), M(100, 64), 0, P, 1 << 40, None)):
        assert rc == g.GOCKPT_EINVAL and text in said(), said()


def test_head_sizes_and_more_refusals():
    L = model._lib()
    h = head()
    rc, need = size("gockpt_head_loss_bytes", h)
    assert rc == 0 and need % 256 == 0 and need > 0
    # columns that products cannot read in place are copied: both matrices, 16 bits, whole pieces of 8
    rc, copied = size("gockpt_head_loss_bytes", head(M(6, 61), M(100, 61)))
    assert rc == 0 and copied == need + 6 * 64 * 2 + 100 * 64 * 2
    assert size("gockpt_head_loss_bytes", head(M(6, 64, 65), M(100, 64, 72)))[1] == need + 6 * 64 * 2
    gx, gw = M(6, 64), M(100, 64)
    assert L.gockpt_head_loss(None, 0, P, P, P, P, need, None) == g.GOCKPT_EINVAL
    assert L.gockpt_head_loss(h, 3, P, P, P, P, need, None) == g.GOCKPT_EINVAL and "reduction 3" in said()
    assert L.gockpt_head_loss(h, -1, P, P, P, P, need, None) == g.GOCKPT_EINVAL
    assert L.gockpt_head_loss(h, 0, P + 2, None, None, P, need, None) == g.GOCKPT_EINVAL
    assert L.gockpt_head_loss(head(classes=200), 0, P, P, P, P, need, None) == g.GOCKPT_EINVAL
    assert "range of the classes" in said()
    assert L.gockpt_head_loss(h, 0, P, P, P, None, 0, None) == g.GOCKPT_EINVAL
    assert L.gockpt_head_loss(h, 0, P, P, P, P + 128, need, None) == g.GOCKPT_EINVAL
    assert L.gockpt_head_loss(h, 0, P, P, P, P, need - 1, None) == g.GOCKPT_ENOMEM
    assert L.gockpt_head_loss_bytes(h, None) == g.GOCKPT_EINVAL
    assert L.gockpt_head_loss(h, 0, None, None, None, P, need, None) == 0  # nothing wanted: no launch
    rc, need = size("gockpt_head_grad_bytes", h, gx, gw)
    assert rc == 0 and need % 256 == 0
    for bad in ((None, 0, P), (P, 0, None), (P + 2, 0, P), (P, 7, P)):
        assert L.gockpt_head_grad(h, *bad, gx, gw, 0, P, need, None) == g.GOCKPT_EINVAL
    for x, w in ((M(5, 64), gw), (M(6, 63), gw), (gx, M(99, 64)), (gx, M(100, 32, 64)), (M(6, 64, 10), gw),
                 (gx, M(100, 64, dtype=3)), (gx, M(100, 64, data=0))):
        assert L.gockpt_head_grad(h, P, 0, P, x, w, 0, P, need, None) == g.GOCKPT_EINVAL
        assert size("gockpt_head_grad_bytes", h, x, w)[0] == g.GOCKPT_EINVAL
    assert L.gockpt_head_grad(h, P, 0, P, gx, gw, 0, P, need - 1, None) == g.GOCKPT_ENOMEM
    assert L.gockpt_head_grad(h, P, 0, P, None, None, 0, P, need, None) == 0  # nothing wanted
    none = head(M(0, 64, data=0), ids=(0, 0, 3, 3, 0, 64, 0))
    assert L.gockpt_head_grad(none, None, 0, None, M(0, 64, data=0), gw, 1, P, need, None) == 0  # nothing to add


def test_the_gradients_workspace_is_bounded():
    """More logits than a piece: Z stays within 256 MiB, or 256 columns."""
    for tokens, rows, cols in ((16384, 50304, 2048), (131072, 131072, 1024), (1 << 20, 131072, 64), (300, 1 << 20, 512)):
        h = head(M(tokens, cols), M(rows, cols), ids=(P, 1, tokens, tokens, 0, 64, 0))
        rc, need = size("gockpt_head_grad_bytes", h, M(tokens, cols), M(rows, cols))
        z = max(256 << 20, tokens * 512)
        # the hidden rows, their fp32 sums (within 256 MiB beyond one slice), slices of a piece's table rows, lists
        assert rc == 0 and need <= z + tokens * cols * 2 + max(256 << 20, tokens * cols * 4) + (1 << 31), need
    logits = 16384 * 50304 * 2
    h = head(M(16384, 2048), M(50304, 2048), ids=(P, 1, 16384, 16384, 0, 64, 0))
    assert size("gockpt_head_grad_bytes", h, M(16384, 2048), M(50304, 2048))[1] < logits / 2
    assert size("gockpt_head_loss_bytes", h)[1] < logits / 20


def A(rows, cols, codes=P, scales=P):
    return model.ACT8.pack(codes, scales, rows, cols)


def test_act8_and_gate_refusals():
    L = model._lib()
    x, a = M(5, 70), A(5, 70)
    for f in (lambda x, a: L.gockpt_act8_pack(x, a, None), lambda x, a: L.gockpt_act8_unpack(a, x, None),
              lambda x, a: L.gockpt_gate8(0, x, None, x, a, None, None),
              lambda x, a: L.gockpt_gate8_grad(0, x, a, None, x, None, None)):
        for bx, ba, text in ((None, a, "null"), (M(5, 70, dtype=4), a, "dtype 4"), (M(5, 70, 69), a, "stride 69"),
                             (M(5, 70, data=0), a, "null"), (M(5, 70, data=P + 1), a, "aligned"),
                             (x, A(4, 70), "4 x 70"), (x, A(5, 96), "5 x 96"), (x, A(5, 70, codes=0), "null"),
                             (x, A(5, 70, codes=P + 8), "16 bytes"), (x, A(5, 70, scales=0), "null")):
            assert f(bx, ba) == g.GOCKPT_EINVAL and text in said(), (text, said())
        empty = M(0, 70, data=0)
        assert f(empty, A(0, 70, 0, 0)) == 0
        assert f(M(5, 0, data=0), A(5, 0, 0, 0)) == 0
    assert L.gockpt_act8_pack(x, None, None) == g.GOCKPT_EINVAL
    gate, back = L.gockpt_gate8, L.gockpt_gate8_grad
    for kind in (-1, 3):
        assert gate(kind, x, None, x, None, None, None) == g.GOCKPT_EINVAL and f"kind {kind}" in said()
        assert back(kind, x, a, None, x, None, None) == g.GOCKPT_EINVAL
    for other in (M(5, 71), M(6, 70), M(5, 70, dtype=FP32), M(5, 70, dtype=9)):
        assert gate(0, x, other, x, None, None, None) == g.GOCKPT_EINVAL
        assert gate(0, x, None, other, None, None, None) == g.GOCKPT_EINVAL
        assert back(0, x, a, None, other, None, None) == g.GOCKPT_EINVAL
        assert back(0, x, a, a, x, other, None) == g.GOCKPT_EINVAL
    # what is kept goes with what there is
    assert gate(0, x, None, x, a, a, None) == g.GOCKPT_EINVAL
    assert gate(0, x, x, x, a, None, None) == g.GOCKPT_EINVAL
    assert gate(0, x, x, x, None, a, None) == g.GOCKPT_EINVAL
    assert back(0, x, a, None, x, x, None) == g.GOCKPT_EINVAL and "without keep_factor" in said()
    assert back(0, x, None, None, x, None, None) == g.GOCKPT_EINVAL
    assert back(0, x, a, a, None, None, None) == 0  # nothing wanted


def test_linear8_refusals():
    L = model._lib()
    x, w, out, keep = M(6, 64), M(32, 64), M(6, 32), A(6, 64)
    rc, need = size("gockpt_linear8_bytes", x, w)
    assert rc == 0
    full = max(need, 256)
    for bx, bw, text in ((None, w, "null x"), (x, None, "null weight"), (M(6, 64, dtype=FP32), w, "x dtype 2"),
                         (x, M(32, 64, dtype=FP16), "x of dtype 0, weight of 1"), (x, M(32, 65), "columns"),
                         (M(6, 64, 60), w, "stride 60"), (x, M((1 << 22) + 1, 64), "rows")):
        assert size("gockpt_linear8_bytes", bx, bw)[0] == g.GOCKPT_EINVAL and text in said(), said()
        assert L.gockpt_linear8(bx, bw, out, keep, P, full, None) == g.GOCKPT_EINVAL
    for o, k in ((None, keep), (M(6, 33), keep), (M(5, 32), keep), (M(6, 32, dtype=3), keep), (out, A(6, 65)),
                 (out, A(5, 64)), (out, A(6, 64, codes=P + 4))):
        assert L.gockpt_linear8(x, w, o, k, P, full, None) == g.GOCKPT_EINVAL
    odd = M(6, 63), M(32, 63)
    rc, need = size("gockpt_linear8_bytes", *odd)
    assert rc == 0 and need >= (6 + 32) * 64 * 2
    assert L.gockpt_linear8(*odd, out, None, P, need - 1, None) == g.GOCKPT_ENOMEM
    assert L.gockpt_linear8(*odd, out, None, None, 0, None) == g.GOCKPT_EINVAL
    assert L.gockpt_linear8(*odd, out, None, P + 64, need, None) == g.GOCKPT_EINVAL
    dy, gx, gw = M(6, 32), M(6, 64), M(32, 64)
    for args in ((None, w, keep, gx, gw), (dy, None, keep, gx, gw), (dy, w, None, gx, gw), (M(6, 32, dtype=FP32), w, keep, gx, gw),
                 (dy, M(32, 64, dtype=FP16), keep, gx, gw), (dy, M(33, 64), keep, gx, gw), (dy, w, keep, M(5, 64), gw),
                 (dy, w, keep, M(6, 63), gw), (dy, w, A(6, 60), gx, gw), (dy, w, A(7, 64), gx, gw),
                 (dy, w, keep, gx, M(31, 64)), (dy, w, keep, gx, M(32, 64, 8)), (dy, w, keep, gx, M(32, 64, dtype=7))):
        assert size("gockpt_linear8_grad_bytes", *args)[0] == g.GOCKPT_EINVAL
        assert L.gockpt_linear8_grad(*args, 0, P, 1 << 40, None) == g.GOCKPT_EINVAL
    # nothing to do: no launch
    assert L.gockpt_linear8_grad(dy, w, keep, None, None, 0, P, 1 << 20, None) == 0
    none = M(0, 64, data=0)
    assert L.gockpt_linear8(none, w, M(0, 32, data=0), A(0, 64, 0, 0), P, 1 << 20, None) == 0
    for f in (L.gockpt_linear8_bytes, ):
        assert f(x, w, None) == g.GOCKPT_EINVAL
    assert L.gockpt_linear8_grad_bytes(dy, w, keep, gx, gw, None) == g.GOCKPT_EINVAL


def test_tensors_off_the_gpu_are_refused():
    import torch
    x, w, y = torch.zeros(4, 8).bfloat16(), torch.zeros(6, 8).bfloat16(), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: g.linear_cross_entropy(x, w, y), lambda: g.head_stats(x, w, y), lambda: g.linear8(x, w),
                 lambda: g.gate8(x), lambda: g.act8_pack(x), lambda: g.Act8((4, 8), x.dtype, "cpu").unpack(),
                 lambda: g.linear8_grad_weight(x, g.Act8((4, 8), x.dtype, "cpu"), torch.zeros(8, 8))):
        with pytest.raises(ValueError):
            call()


def test_8_bits_take_33_bytes_for_32():
    import torch
    a = g.Act8((3, 5, 100), torch.bfloat16, "cpu")
    assert a.codes.shape == (15, 128) and a.scales.shape == (15, 4) and a.nbytes == 15 * 4 * 33
    assert struct.calcsize(model.ACT8.format) == 32
    with pytest.raises(ValueError):
        g.Act8((), torch.bfloat16, "cpu")
    with pytest.raises(ValueError):
        g.Act8((3,), torch.int8, "cpu")


def test_products_of_more_blocks_than_a_grid_are_refused():
    L = model._lib()
    # 2^30 tokens and 2^22 classes of 8 columns: 2^22 x 2^14 tiles of 256 x 256
    n = 1 << 30
    h = head(M(n, 8), M(1 << 22, 8), ids=(P, 1, n, n, 0, 64, 0))
    rc, need = size("gockpt_head_loss_bytes", h)
    assert rc == g.GOCKPT_EINVAL and need == 0 and "tiles" in said()
    assert L.gockpt_head_loss(h, 0, P, P, P, P, 1 << 62, None) == g.GOCKPT_EINVAL
    x, w = M(n, 8), M(1 << 22, 8)
    assert size("gockpt_linear8_bytes", x, w)[0] == g.GOCKPT_EINVAL and "tiles" in said()
    assert L.gockpt_linear8(x, w, M(n, 1 << 22), None, P, 1 << 62, None) == g.GOCKPT_EINVAL


def test_copies_are_made_on_the_calls_stream(monkeypatch):
    import torch
    seen = []

    class Now:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            seen.append(self.stream)

        def __exit__(self, *a):
            seen.append("out")

    monkeypatch.setattr(torch.cuda, "stream", Now)
    t = torch.zeros(6, 4).t()
    own = model._own_rows(t, 6, "s")
    assert own.is_contiguous() and seen == ["s", "out"]
    rows = torch.zeros(4, 8)[:, :6]
    assert model._own_rows(rows, 6, "s") is rows and len(seen) == 2


def test_a_copy_of_8_bits_has_its_own_address():
    """copy.deepcopy and pickle give a copy another buffer; what the library is given names that one."""
    import copy
    import pickle

    import torch
    a = g.Act8((3, 40), torch.bfloat16, "cpu")
    a.buffer.copy_(torch.arange(a.nbytes).to(torch.uint8))
    for b in (copy.deepcopy(a), pickle.loads(pickle.dumps(a)), copy.deepcopy([a, a])[1]):
        assert b.buffer.data_ptr() != a.buffer.data_ptr() and b.shape == a.shape and b.dtype == a.dtype
        assert torch.equal(b.codes, a.codes) and torch.equal(b.scales, a.scales)
        # nothing in it but the buffer says where that lies
        at = (a.buffer.data_ptr(), a.buffer.data_ptr() + 3 * 64)
        for name in b.__slots__:
            held = getattr(b, name)
            assert not isinstance(held, bytes) or not any(struct.pack("<Q", x) in held for x in at), name
        assert model.ACT8.unpack(b._at(b.buffer)) == (b.buffer.data_ptr(), b.buffer.data_ptr() + 3 * 64, 3, 40)
    shallow = copy.copy(a)  # the same memory, as a shallow copy of a tensor is
    assert shallow.buffer is a.buffer


def test_products_of_more_threads_than_a_launch_has_are_refused():
    """A launch has fewer than 2^32 threads: 2^23 - 1 blocks of 512, a tile of 256 x 256 each."""
    L = model._lib()
    for tokens, rows, ok in ((1 << 22, 131072, False), ((1 << 22) - 256, 131072, True), (1 << 22, 131072 - 256, True),
                             (1 << 23, 65536, False), (1 << 23, 65537, False), (1 << 26, 16384, False)):
        h = head(M(tokens, 64), M(rows, 64), ids=(P, 1, tokens, tokens, 0, 64, 0))
        rc, need = size("gockpt_head_loss_bytes", h)
        assert (rc == 0) == ok and (need > 0) == ok, (tokens, rows, rc)
        x, w = M(tokens, 64), M(rows, 64)
        rc8, need8 = size("gockpt_linear8_bytes", x, w)
        assert (rc8 == 0) == ok, (tokens, rows, rc8)
        if ok:  # and with too little workspace nothing is launched
            assert L.gockpt_head_loss(h, 0, P, P, P, P, need - 1, None) == g.GOCKPT_ENOMEM
            continue
        assert rc == rc8 == g.GOCKPT_EINVAL and need8 == 0 and "tiles" in said()
        # before anything is launched
        assert L.gockpt_head_loss(h, 0, P, P, P, P, 1 << 62, None) == g.GOCKPT_EINVAL and "tiles" in said()
        assert L.gockpt_linear8(x, w, M(tokens, rows), A(tokens, 64), P, 1 << 62, None) == g.GOCKPT_EINVAL
        # the same product as an input's gradient, and as a weight's
        dy, wide = M(tokens, 64), M(64, rows)
        for args in ((dy, wide, None, M(tokens, rows), None),):
            assert size("gockpt_linear8_grad_bytes", *args)[0] == g.GOCKPT_EINVAL and "tiles" in said()
            assert L.gockpt_linear8_grad(*args, 0, P, 1 << 62, None) == g.GOCKPT_EINVAL
    # the head's gradients take the vocabulary in pieces, whose products are small enough
    n = 1 << 22
    h = head(M(n, 64), M(131072, 64), ids=(P, 1, n, n, 0, 64, 0))
    assert size("gockpt_head_grad_bytes", h, M(n, 64), M(131072, 64))[0] == 0
    n = 1 << 30  # 2^22 tiles of tokens
    h = head(M(n, 512), M(131072, 512), ids=(P, 1, n, n, 0, 64, 0))
    assert size("gockpt_head_grad_bytes", h, M(n, 512), None)[0] == g.GOCKPT_EINVAL and "tiles" in said()
