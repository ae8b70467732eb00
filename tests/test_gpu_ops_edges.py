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
