"""A row of cross attention is its own: the same bits whatever the other sequences' queries are, and whatever a
kernel before has left where a tile of 128 rows has none (three, five or seven heads a KV head)."""
import pytest
import torch

from test_cross_gpu import Case

pytestmark = pytest.mark.gpu


def bits(x):
    return x.contiguous().view(torch.int16 if x.dtype != torch.float32 else torch.int32)


@pytest.mark.parametrize("per", [1, 3, 4, 5, 7])
@pytest.mark.parametrize("n,states", [(1, 300), (9, 300), (50, 700), (130, 300), (45, 3000)])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f16")])
def test_rows_are_their_own(n, states, per, d, dtype):
    c = Case(61 + n, [n, n, n], [states, states // 2, states], 2, per, d, dtype)
    loud = Case(62, [n] * 3, [states, states // 2, states], 2, per, d, dtype, scale=64.0)
    o, lse = c.forward()
    grads = c.backward(o, lse)
    mine = slice(n, 2 * n)
    q = c.q.clone()
    for size in (0.0, 4.0, 300.0, float("nan")):
        c.q[:n], c.q[2 * n:] = q[:n] * size, q[2 * n:] * size
        loud.q.copy_(q * (size if size == size else 1e4))
        loud.backward(*loud.forward())
        o2, lse2 = c.forward()
        assert torch.equal(bits(o2[mine]), bits(o[mine])) and torch.equal(bits(lse2[mine]), bits(lse[mine]))
        g2 = c.backward(o2, lse2)
        rows = slice(c.kb[1], c.kb[2])
        for a, b, s in zip(g2, grads, (mine, rows, rows)):
            assert torch.equal(bits(a[s]), bits(b[s]))
