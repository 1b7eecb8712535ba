"""Attention's tensors are looked over before a stream, a capture or a workspace is asked for: on a machine without
a device, too, each refusal names what is wrong, and no workspace is made for a call that is refused."""
import pytest
import torch

from paper_2607_29591_gb300 import build as B
from paper_2607_29591_gb300 import reskv as R


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()
    R._calls()


class Held:
    """A cache's shape without memory."""
    batch, table_pages, n_kv_heads, head_dim, address = 2, 3, 2, 128, 0
    attn_workspace = {}

    @property
    def struct(self):
        raise AssertionError("a refused call asks for no workspace's size")


def rows(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def ints(n):
    return torch.zeros(n, dtype=torch.int32)


def test_paged_attention():
    before = dict(R._workspaces)
    with pytest.raises(ValueError, match="q must be a CUDA tensor"):
        R.reskv_paged_attn(Held(), rows(2, 4, 128), ints(2), rows(2, 4, 128))
    with pytest.raises(ValueError, match="q must be a CUDA tensor"):
        R.reskv_paged_attn_shared(Held(), Held(), rows(2, 4, 128), ints(2), ints(2), rows(2, 4, 128))
    assert R._workspaces == before


@pytest.mark.parametrize("q,k,word", [(rows(3, 4, 64), rows(5, 2, 64), "q must be a CUDA tensor"), (rows(3), rows(5, 2, 64), "tokens, heads, dim"),
                                      (rows(3, 64), rows(5, 2, 64), "tokens, heads, dim"), (rows(3, 4, 64), rows(64), "tokens, heads, dim")])
def test_the_gradient_of_cross_attention(q, k, word):
    before = dict(R._workspaces)
    with pytest.raises(ValueError, match=word):
        R.reskv_cross_attn_backward(q, k, k, q, torch.zeros((3, 4)), q, q, k, k)
    with pytest.raises(ValueError, match="lse"):
        R.reskv_cross_attn_backward(q, k, k, q, None, q, q, k, k)
    assert R._workspaces == before
