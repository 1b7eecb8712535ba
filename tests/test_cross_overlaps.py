"""Gradients of cross attention that would lie over what is still read are refused (no GPU needed)."""
import pytest

from paper_2607_29591_gb300 import build as B
from paper_2607_29591_gb300 import reskv as R

P = 1 << 20


@pytest.fixture(scope="module")
def lib():
    B.build()
    return R.load_library()


def call(lib, **at):
    """Tensors at addresses of their own, but for those of `at` (by name: another's name)."""
    names = ["q", "k", "v", "o", "d_o", "d_q", "d_k", "d_v"]
    where = {n: P * (i + 2) for i, n in enumerate(names)}
    where.update({n: where[x] for n, x in at.items()})
    t = {n: R.reskv_heads(where[n], 1024, 128, 2 if n in ("k", "v", "d_k", "d_v") else 8, R.RESKV_BF16) for n in names}
    a = R.reskv_cross_attn_args(q=t["q"], k=t["k"], v=t["v"], o=t["o"], lse=P, n_tokens=10, n_rows=20, batch=1, head_dim=128,
                                workspace=P, workspace_bytes=1 << 19)
    return lib.reskv_cross_attn_backward(a, t["d_o"], t["d_q"], t["d_k"], t["d_v"], None)


@pytest.mark.parametrize("which,over", [("d_q", "q"), ("d_q", "d_o"), ("d_q", "k"), ("d_q", "v"), ("d_k", "q"), ("d_v", "q"), ("d_k", "d_o"),
                                        ("d_v", "d_o"), ("d_k", "d_q"), ("d_v", "d_q"), ("d_v", "d_k")])
def test_refused(lib, which, over):
    assert call(lib, **{which: over}) == R.RESKV_ERR_INVALID_ARG and "must not lie over" in R.reskv_last_error()
