"""Logits of -inf in cross attention (products past fp32): such a state has weight 0, wherever it lies, and a query
all of whose logits are -inf is one that sees nothing.  The others' values and gradients are those without the states."""
import numpy as np
import pytest
import torch

from oracle import cross_oracle as co
from paged_cases import HALF_ULP
from test_cross_gpu import LEAST, Case, check

pytestmark = pytest.mark.gpu

FORMS = [(1, [300, 40], 0), (3, [2000, 130], 0), (40, [300, 40], 0), (150, [300, 40], 0), (20, [2000, 300], 0), (2, [60, 40], 1), (9, [60, 40], 1)]


def far_case(n, lens, offset, d, where):
    """Sequence 0's states `where` and all of sequence 1's have logits of -inf with every query."""
    c = Case(71 + n, [n, n], lens, 2, 2, d, "bf16", offset=offset)
    c.q[:, :, 0] = c.q[:, :, 0].abs() + 2
    rows = torch.tensor([c.kb[0] + w for w in where] + list(range(c.kb[1], c.kb[2])), device="cuda")
    c.k[rows] = 0
    c.k[rows, :, 0] = -3e38
    c.q64, c.k64 = c.q.double().cpu().numpy(), c.k.double().cpu().numpy()
    c.near = np.array([i for i in range(lens[0]) if i not in where])
    return c


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,lens,offset", FORMS)
@pytest.mark.parametrize("where", [[0], [1, 2, 3], list(range(50)), [0, 39]])
def test_states_of_no_weight(where, n, lens, offset, d):
    c = far_case(n, lens, offset, d, where)
    o, lse = c.forward()
    t, r = slice(0, n), c.kb[0] + c.near
    k, v = c.k64[r].transpose(1, 0, 2), c.v64[r].transpose(1, 0, 2)
    check(o[t], lse[t], [co.attend(c.q64[t], k, v, d ** -0.5)], d, "bf16")
    assert (o[n:] == 0).all() and (lse[n:] == -np.inf).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,lens,offset", FORMS)
@pytest.mark.parametrize("where", [[0], [1, 2, 3], [0, 39]])
def test_gradients_without_them(where, n, lens, offset, d):
    c = far_case(n, lens, offset, d, where)
    dq, dk, dv = (x.double().cpu().numpy() for x in c.backward(*c.forward()))
    t, r = slice(0, n), c.kb[0] + c.near
    ref, tol = co.gradient(c.q64[t], c.k64[r].transpose(1, 0, 2), c.v64[r].transpose(1, 0, 2), c.g64[t], d ** -0.5,
                           HALF_ULP["bf16"], LEAST["bf16"])
    for got, want, off in ((dq[t], ref[0], tol[0]), (dk[r].transpose(1, 0, 2), ref[1], tol[1]), (dv[r].transpose(1, 0, 2), ref[2], tol[2])):
        assert np.isfinite(got).all() and (np.abs(got - want) <= off * 1.01).all()
    gone = np.setdiff1d(np.arange(c.rows), r)
    assert (dk[gone] == 0).all() and (dv[gone] == 0).all() and (dq[n:] == 0).all()
