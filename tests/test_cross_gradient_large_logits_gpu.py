"""The gradient of cross attention where logits are large: the log-sum-exp that it is given is then off by far more
than a weight's digits, as fp32 holds it, and weights are formed from the row's own logits instead."""
import numpy as np
import pytest
import torch

from oracle import cross_oracle as co
from paged_cases import HALF_ULP
from test_cross_gpu import LEAST, Case

pytestmark = pytest.mark.gpu

FORMS = [([1, 3], [300, 40], 0), ([3], [3000], 0), ([40, 9], [300, 129], 0), ([20, 30], [2100, 700], 0), ([300], [400], 0), ([4, 9], [60, 50], 2)]


def offset_case(counts, lens, d, dtype, size, sign, offset, both=False):
    """Logits `size` + differences of some ones (both: of half of the queries' heads), every partial sum exact in fp32."""
    c = Case(81, counts, lens, 2, 2, d, dtype, scale=float(sign), offset=offset)
    rng = np.random.default_rng(int(np.log2(size)) + d)
    root = 2.0 ** (int(np.log2(size)) // 2)
    q, k = np.zeros(c.q64.shape), np.zeros(c.k64.shape)
    q[..., 1:5] = rng.choice([-1.0, 1.0], q.shape[:-1] + (4,))
    k[..., 1:5] = rng.integers(-8, 9, k.shape[:-1] + (4,)) / 8
    q[..., 0], k[..., 0] = sign * root, size / root
    if both:
        q[:, 1::2, 0] = 0
    c.q.copy_(torch.from_numpy(q))
    c.k.copy_(torch.from_numpy(k))
    c.q64, c.k64 = c.q.double().cpu().numpy(), c.k.double().cpu().numpy()
    assert (c.q64 == q).all() and (c.k64 == k).all()
    return c


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("counts,lens,offset", FORMS)
@pytest.mark.parametrize("size,sign,both", [(2.0 ** 6, 1, False), (2.0 ** 8, 1, False), (2.0 ** 9, -1, False), (2.0 ** 10, 1, True),
                                            (2.0 ** 13, 1, False), (2.0 ** 16, -1, True), (2.0 ** 20, 1, False), (2.0 ** 20, 1, True)])
def test_a_common_offset(size, sign, both, counts, lens, offset, dtype, d):
    c = offset_case(counts, lens, d, dtype, size, sign, offset, both)
    dq, dk, dv = (x.double().cpu().numpy() for x in c.backward(*c.forward()))
    assert int(c.status) == 0
    for b, (t, r, _) in enumerate(c.sequences()):
        ref, tol = co.gradient_norms(c.q64[t], c.k64[r].transpose(1, 0, 2), c.v64[r].transpose(1, 0, 2), c.g64[t], c.scale,
                                     HALF_ULP[dtype], LEAST[dtype], exact=True)
        n = t.stop - t.start
        heads = lambda x: x.reshape(n, 2, 2, d).transpose(1, 0, 2, 3)  # noqa: E731
        for i, (got, want) in enumerate(((heads(dq[t]), heads(ref[0])), (dk[r].transpose(1, 0, 2), ref[1]), (dv[r].transpose(1, 0, 2), ref[2]))):
            for h in range(2):
                # (of d_q without the dim that all keys share: a sum of 0 times their size, which keeps the products of
                # T's and P's roundings)
                a, w = (got[h][..., 1:], want[h][..., 1:]) if i == 0 else (got[h], want[h])
                off = np.linalg.norm(a - w)
                assert off <= tol[i, h], (b, i, h, off, tol[i, h], np.linalg.norm(w))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("counts,lens,offset", FORMS)
@pytest.mark.parametrize("dtype,size", [("bf16", s) for s in (1e3, 1e5, 1e7, 1e9, 1e12, 1e20, 1e30)] + [("f16", 1e3), ("f16", 3e4)])
def test_equal_winners_share(dtype, size, counts, lens, offset, d):
    """Three equal keys whose logits are far above all others': a third of the weight each.  d_v and d_k of the
    three are known, all others are 0; d_q, the same key times a sum of T that is 0, keeps e (1 - sum P) of it, as rounded:
    e, the rounded sum of T, is what D lacks (HALF_ULP sum |d_o o|) and T's roundings, 1 - sum P at most HALF_ULP."""
    c = Case(82, counts, lens, 1, 4, d, dtype, offset=offset)
    g = torch.Generator(device="cuda").manual_seed(5)
    c.q.copy_(1 + 0.1 * torch.rand(c.q.shape, generator=g, device="cuda"))
    if dtype == "f16" and size > 1e3:
        c.q.mul_(1024)
    c.k.mul_(0.01)
    wins = []
    for b, (t, r, _) in enumerate(c.sequences()):
        w = [r.start, r.start + lens[b] // 2, r.stop - 1]
        c.k[w] = (size * (1 + torch.rand(d, generator=g, device="cuda"))).to(c.k.dtype)
        wins.append(w)
    c.q64, c.k64 = c.q.double().cpu().numpy(), c.k.double().cpu().numpy()
    grads = c.backward(*c.forward())
    dq, dk, dv = (x.double().cpu().numpy() for x in grads)
    assert int(c.status) == 0
    unit, scale = HALF_ULP[dtype], d ** -0.5
    for b, (t, r, _) in enumerate(c.sequences()):
        w = wins[b]
        gg, qq, vv, kk = c.g64[t], c.q64[t], c.v64[w][:, 0], c.k64[w[0], 0]
        G = gg @ vv.T                                       # [n, H, 3]
        T = (G - G.mean(-1, keepdims=True)) / 3
        off = np.abs(gg) @ np.abs(vv).T * 2.0 ** -16         # fp32 sums, P's last digits
        for j in range(3):
            want = gg.sum((0, 1)) / 3
            tol = (np.abs(gg).sum((0, 1)) / 3) * (unit + 2.0 ** -12) + unit * np.abs(want) * 1.01 + LEAST[dtype] * gg.size
            assert (np.abs(dv[w[j], 0] - want) <= tol).all(), (b, j, "dv")
            want = scale * (T[..., j, None] * qq).sum((0, 1))
            t_off = np.abs(T[..., j]) * (unit + 2.0 ** -12) + off[..., j] + LEAST[dtype]
            tol = scale * (t_off[..., None] * np.abs(qq)).sum((0, 1)) + unit * np.abs(want) * 1.01 + LEAST[dtype]
            assert (np.abs(dk[w[j], 0] - want) <= tol * 1.01).all(), (b, j, "dk")
        rest = np.setdiff1d(np.arange(r.start, r.stop), w)
        assert (dk[rest] == 0).all() and (dv[rest] == 0).all()
        lost = (np.abs(gg) * np.abs(vv).mean(0)).sum(-1) * unit + off.sum(-1)      # of D, by the rounding of o
        spare = ((np.abs(T) * unit).sum(-1) + lost) * (unit + 2.0 ** -12) + 2.0 ** -20 * off.sum(-1) + 3 * LEAST[dtype]
        tol = scale * spare[..., None] * np.abs(kk) + LEAST[dtype]
        assert (np.abs(dq[t]) <= tol).all(), (b, "dq", np.abs(dq[t] / kk).max(), (tol / np.abs(kk)).min())
