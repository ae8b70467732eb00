"""Edges of the model's operators on the GPU.  Tolerances as in test_gpu_model,
whose helpers these tests take."""
import copy
import pickle

import pytest

import paper_2511_07035_amd as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_model import DT, assert_close, kept64, product_error, randn  # noqa: E402


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
