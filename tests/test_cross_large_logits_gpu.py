"""Cross attention whose logits are past what fp32 counts in ones: few query rows, many, and rows of any alignment.

Tolerances: equal keys have equal logits, bit for bit, so that m of them share the weight and the others have none.
A weight is rounded to q's type (HALF_ULP of it; the reference of a row's weights is a power of two), the sums
are fp32, the output is rounded: an output is off by HALF_ULP times the mean |v| of the winners, then HALF_ULP of itself.
The log-sum-exp is the logit, d products and a scaling of fp32, and ln m."""
import numpy as np
import pytest
import torch

from paged_cases import DT, HALF_ULP
from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


def keys_and_queries(size, n, states, winners, d, dtype, seed, kv=1, per=4):
    """Keys whose products with all queries are near size * d * scale at the winners, minus that at one other, and small."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = 0.1 * torch.randn((states, kv, d), generator=g, device="cuda")
    k[winners] = size * (1 + torch.rand((1, kv, d), generator=g, device="cuda"))
    k[[i for i in range(5, 200) if i not in winners][0]] = -2 * size
    v = torch.randn((states, kv, d), generator=g, device="cuda")
    q = 1 + 0.1 * torch.rand((n, kv * per, d), generator=g, device="cuda")
    return q.to(DT[dtype]), k.to(DT[dtype]), v.to(DT[dtype])


SIZES = [("bf16", s) for s in (1e2, 1e4, 1e5, 1e7, 1e8, 3e8, 1e9, 1e10, 1e12, 1e15, 1e20, 1e30)] + [("f16", s) for s in (1e2, 1e4, 3e4)]
FORMS = [(1, 300, 0), (4, 4000, 0), (3, 300, 1), (5, 300, 0), (40, 300, 0), (30, 2000, 0), (150, 400, 0)]


def place(t, offset):
    flat = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
    flat[offset:] = t.flatten()
    return flat[offset:].view(t.shape)


@pytest.mark.parametrize("n,states,offset", FORMS)
@pytest.mark.parametrize("dtype,size", SIZES)
@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_equal_winners_share(d, many, dtype, size, n, states, offset):
    winners = [states // 3] + ([0, 70, 131, 200, states - 1] if many else [])
    q, k, v = keys_and_queries(size, n, states, winners, d, dtype, n)
    big = 1024.0 if dtype == "f16" else 1.0                 # (fp16's keys end early: logits of 1e10 by large queries)
    q = q * big if size >= 1e4 else q
    q, k, v = (place(x, offset) for x in (q, k, v))
    o, lse = torch.full_like(q, float("nan")), torch.empty(q.shape[:2], device="cuda")
    R.reskv_cross_attn(q, k, v, o, lse=lse)
    w = v[winners].double()                                 # [m, 1, d]
    mean = w.mean(0)
    tol = HALF_ULP[dtype] * w.abs().mean(0) + HALF_ULP[dtype] * mean.abs() * 1.01 + 2.0 ** -16
    assert torch.isfinite(o).all()
    assert ((o.double() - mean).abs() <= tol).all()
    logit = (q.double() * k[winners[0]].double()).sum(-1) * d ** -0.5
    assert ((lse.double() - logit - np.log(len(winners))).abs() <= (d + 1) * 2.0 ** -23 * logit.abs() + 2.0 ** -16).all()


@pytest.mark.parametrize("n", [2, 40])
def test_rows_near_the_end_of_fp16(n):
    """Every element near 2e4: logits of 4.5e9 that lie some 1e6 apart."""
    g = torch.Generator(device="cuda").manual_seed(n)
    q = (20000 + 16 * torch.randint(-2, 3, (n, 4, 128), generator=g, device="cuda")).half()
    k = (20000 + 16 * torch.randint(-2, 3, (500, 1, 128), generator=g, device="cuda")).half()
    k[77] = 20112
    v = torch.randn((500, 1, 128), generator=g, device="cuda").half()
    o = torch.empty_like(q)
    R.reskv_cross_attn(q, k, v, o)
    assert torch.equal(o, v[77].expand_as(o))


@pytest.mark.parametrize("n", [2, 40])
@pytest.mark.parametrize("per_unit", [2.0 ** 20, 2.0 ** 23, 2.0 ** 24])
def test_logits_that_climb_in_small_steps(n, per_unit):
    """Logits of 2^24 to 2^28 whose tiles' largest climb by some fp32 steps each: one output row is one value's."""
    states = 1300
    q = torch.full((n, 2, 64), 1024.0, device="cuda").half()
    k = torch.zeros((states, 1, 64), device="cuda")
    k[:, :, 0] = per_unit * 2.0 ** -10                      # 1024 times that each
    k[:, :, 1] = torch.arange(states, device="cuda")[:, None] / 8.0
    k = k.clamp(max=60000).half()
    v = torch.randn((states, 1, 64), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").half()
    o, lse = torch.empty_like(q), torch.empty((n, 2), device="cuda")
    for scale in (1.0, 0.5, 0.3):
        R.reskv_cross_attn(q, k, v, o, scale=scale, lse=lse)
        assert torch.isfinite(o).all() and torch.isfinite(lse).all()
        assert float((o.double() - v[-1].double()).abs().max()) <= 2.0 ** -10 * 5      # the last key's logit is 38 above the next's
