"""What the bound on the norms of cross attention's gradients (oracle.cross_oracle.gradient_norms) refuses: D = <d_o, o>
left out, half of it, and where attention has a peak D of the o that 16 bits hold.  The mistakes are the oracle's own."""
import numpy as np
import pytest

from oracle import cross_oracle as co

HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25}


def inputs(n, length, d, per=4, akin=0.0):
    rng = np.random.default_rng(n + length)
    q, g = rng.standard_normal((2, n, per, d))
    k, v = rng.standard_normal((2, 1, length, d))
    if akin:
        q = (1 - akin) * q + akin * 8 * k[0, rng.integers(0, length, (n, per))] / np.sqrt(d) * 4
    return q, k, v, g


def rounded(x, dtype):
    if dtype == "f16":
        return x.astype(np.float16).astype(np.float64)
    m, e = np.frexp(x)
    return np.ldexp(np.round(m * 256) / 256, e)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,length", [(1, 100), (3, 129), (20, 100), (100, 100), (100, 1000), (20, 2100), (257, 127)])
def test_a_missing_term_is_refused(n, length, dtype):
    q, k, v, g = inputs(n, length, 128)
    scale = 128 ** -0.5
    right, tol = co.gradient_norms(q, k, v, g, scale, HALF_ULP[dtype], LEAST[dtype])
    D = (g * co.attend(q, k, v, scale)[0]).sum(-1)
    for share in (0.0, 0.5):
        wrong, _ = co.gradient_norms(q, k, v, g, scale, HALF_ULP[dtype], LEAST[dtype], of_d=share * D)
        for i in range(2):
            assert np.linalg.norm(wrong[i] - right[i]) > 2 * tol[i, 0], (share, i)


@pytest.mark.parametrize("n,length", [(20, 100), (100, 300), (512, 577)])
def test_d_of_the_rounded_output_is_refused_at_a_peak(n, length):
    """Queries akin to a key (most of the weight on it): G - D is small beside D's error."""
    q, k, v, g = inputs(n, length, 64, akin=0.5)
    scale = 64 ** -0.5
    o = co.attend(q, k, v, scale)[0]
    right, tol = co.gradient_norms(q, k, v, g, scale, HALF_ULP["bf16"], LEAST["bf16"])
    wrong, _ = co.gradient_norms(q, k, v, g, scale, HALF_ULP["bf16"], LEAST["bf16"], of_d=(g * rounded(o, "bf16")).sum(-1))
    print(np.linalg.norm(wrong[0] - right[0]) / tol[0, 0], np.linalg.norm(wrong[1] - right[1]) / tol[1, 0],
          tol[0, 0] / np.linalg.norm(right[0]), tol[1, 0] / np.linalg.norm(right[1]))
    assert np.linalg.norm(wrong[0] - right[0]) > tol[0, 0]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,length,akin", [(1, 2, 0), (2, 50, 0), (20, 300, 0.5), (300, 500, 0)])
def test_roundings_alone_pass(n, length, akin, dtype):
    """p, t and the results rounded as the type rounds, all else in 64 bits."""
    q, k, v, g = inputs(n, length, 64, akin=akin)
    scale = 64 ** -0.5
    right, tol = co.gradient_norms(q, k, v, g, scale, HALF_ULP[dtype], LEAST[dtype])
    got = [np.zeros_like(x) for x in right]
    for h in range(q.shape[1]):
        x = scale * (q[:, h] @ k[0].T)
        p = np.exp(x - x.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        t = p * (g[:, h] @ v[0].T - (g[:, h] * (p @ v[0])).sum(1, keepdims=True))
        tr, pr = rounded(t, dtype), rounded(p, dtype)
        got[0][:, h] = scale * (tr @ k[0] - tr.sum(1, keepdims=True) * (pr @ k[0]))
        got[1][0] += scale * (tr.T @ q[:, h])
        got[2][0] += pr.T @ g[:, h]
    for i in range(3):
        assert np.linalg.norm(rounded(got[i], dtype) - right[i]) <= tol[i, 0]
