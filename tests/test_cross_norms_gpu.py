"""The norms of cross attention's gradients against fp64: flat and peaked queries, few and many rows, every form."""
import numpy as np
import pytest
import torch

from cross_cases import check_norms
from test_cross_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("counts,lens", [([1, 2], [50, 300]), ([3], [3000]), ([20, 3], [2100, 700]), ([130, 1, 257], [257, 300, 127]),
                                         ([600], [577])])
def test_flat_queries(counts, lens, d, dtype):
    check_norms(Case(51, counts, lens, 2, 2, d, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,states,d", [(1, 40, 64), (20, 300, 128), (300, 577, 64), (260, 1500, 128)])
def test_queries_akin_to_a_key(n, states, d, dtype):
    """Most of a row's weight on one key: what the rounding of o takes from D would be most of G - D."""
    c = Case(52, [n, n], [states, states + 1], 2, 4, d, dtype)
    rng = np.random.default_rng(n)
    for t, r, _ in c.sequences():
        pick = torch.from_numpy(rng.integers(r.start, r.stop, n)).cuda()
        near = c.k[pick].repeat_interleave(c.per, 1)
        c.q[t] = (1.5 * near.float() + 0.7 * c.q[t].float()).to(c.q.dtype)
    c.q64 = c.q.double().cpu().numpy()
    c.check()
    check_norms(c)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("offset", [1, 4])
@pytest.mark.parametrize("n,states,d", [(1, 40, 64), (20, 100, 128), (40, 200, 64)])
def test_rows_of_any_alignment(n, states, d, offset, dtype):
    """The same for rows off 16-byte boundaries, with queries akin to a key."""
    c = Case(53, [n, n], [states, states + 1], 2, 4, d, dtype, offset=offset)
    rng = np.random.default_rng(n)
    for t, r, _ in c.sequences():
        pick = torch.from_numpy(rng.integers(r.start, r.stop, n)).cuda()
        c.q[t] = (1.5 * c.k[pick].repeat_interleave(c.per, 1).float() + 0.7 * c.q[t].float()).to(c.q.dtype)
    c.q64 = c.q.double().cpu().numpy()
    c.check()
    check_norms(c)
