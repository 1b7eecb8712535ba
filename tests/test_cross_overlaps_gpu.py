"""Gradients of cross attention in the place of what each block alone reads: the same bits."""
import pytest
import torch

from paper_2607_29591_gb300 import reskv as R
from test_cross_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("counts,lens", [([3, 9], [60, 300]), ([300], [400]), ([20], [2000]), ([700], [130])])
def test_gradients_in_place(counts, lens, offset):
    c = Case(111, counts, lens, 2, 2, 64, "bf16", offset=offset if max(lens) < 1000 else 0)
    o, lse = c.forward()
    want = c.backward(o, lse)
    R.reskv_cross_attn_backward(c.q, c.k, c.v, o, lse, c.g, o, c.k, c.v, status=c.status, **c.args)
    for a, b in zip((o, c.k, c.v), want):
        assert torch.equal(a, b)
