"""Rotary positions (reskv_rope, reskv_rope_table) against fp64.

Tolerance of a turned value a c - b s: two rounded products and a rounded sum in
fp32 from an fp32 table, 3 * 2^-24 (|a c| + |b s|) and slack, then half a unit in
the last place of the output type.
"""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paged_cases import DT, HALF_ULP, as_type, rows
from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


def turned(x, cs, interleaved, backward):
    """fp64 result and the sum of magnitudes its rounding scales with."""
    y = po.rotate(x, cs, interleaved, backward)
    size = po.rotate(np.abs(x), np.stack([np.abs(cs[..., 0]), -np.abs(cs[..., 1])], -1), interleaved)
    size2 = po.rotate(np.abs(x), np.abs(cs), interleaved)
    return y, np.maximum(np.abs(size), np.abs(size2))


def check(got, ref, size, dtype):
    err = np.abs(got.double().cpu().numpy() - ref)
    tol = 4 * 2.0 ** -24 * size + HALF_ULP[dtype] * np.abs(ref) * (1 + 2.0 ** -8) + (2.0 ** -25 if dtype == "f16" else 0)
    assert (err <= tol).all(), (err - tol).max()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,K,d,rot", [(1, 32, 8, 128, 128), (7, 3, 1, 128, 64), (33, 4, 2, 64, 32), (5, 2, 2, 96, 96),
                                         (3, 1, 1, 2, 2), (9, 2, 1, 10, 6), (2, 5, 3, 512, 512), (4, 2, 1, 80, 24)])
def test_rotation_matches_fp64(dtype, interleaved, T, H, K, d, rot):
    rng = np.random.default_rng(d * T + rot)
    tab = po.table(50, po.frequencies(rot)).astype(np.float32)
    pos = rng.integers(0, 50, T).astype(np.int32)
    q, q64 = as_type(rows(rng, (T, H), d), dtype)
    k, k64 = as_type(rows(rng, (T, K), d), dtype)
    table, p = torch.from_numpy(tab).cuda(), torch.from_numpy(pos).cuda()
    for backward in (False, True):
        qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
        R.reskv_rope(q, qo, p, table, k=k, k_out=ko, interleaved=interleaved, backward=backward)
        for got, x in ((qo, q64), (ko, k64)):
            check(got, *turned(x, tab[pos].astype(np.float64), interleaved, backward), dtype)
            if rot < d:
                np.testing.assert_array_equal(got.double().cpu().numpy()[..., rot:], x[..., rot:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_backward_is_the_gradient(interleaved):
    """<w, rope(x)> has the gradient rope_backward(w): against central differences of the forward pass."""
    rng = np.random.default_rng(5)
    T, H, d, rot = 3, 2, 16, 8
    table = torch.from_numpy(po.table(9, po.frequencies(rot), 1.25).astype(np.float32)).cuda()
    p = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda")
    x = torch.from_numpy(rng.standard_normal((T, H, d)).astype(np.float32)).cuda()
    w = torch.from_numpy(rng.standard_normal((T, H, d)).astype(np.float32)).cuda()
    grad = torch.empty_like(x)
    R.reskv_rope(w, grad, p, table, interleaved=interleaved, backward=True)

    def value(y):
        out = torch.empty_like(y)
        R.reskv_rope(y, out, p, table, interleaved=interleaved)
        return float((out.double() * w.double()).sum())

    # the map is linear: a central difference of step 1 has rounding errors only
    for i in rng.integers(0, x.numel(), 24):
        e = torch.zeros(x.numel(), device="cuda")
        e[i] = 0.5
        e = e.view_as(x)
        assert abs(value(x + e) - value(x - e) - float(grad.flatten()[i])) < 1e-4


def test_strides_in_place_and_unaligned_rows():
    rng = np.random.default_rng(1)
    tab = po.table(40, po.frequencies(128)).astype(np.float32)
    table = torch.from_numpy(tab).cuda()
    pos = torch.arange(11, dtype=torch.int32, device="cuda") + 3
    fused = torch.from_numpy(rows(rng, (11, 12), 128)).bfloat16().cuda()          # q 8, k 2, v 2 heads
    want = fused.clone()
    qo, ko = (torch.empty((11, h, 128), dtype=torch.bfloat16, device="cuda") for h in (8, 2))
    R.reskv_rope(fused[:, :8], qo, pos, table, k=fused[:, 8:10], k_out=ko)
    assert torch.equal(fused, want)
    R.reskv_rope(fused[:, :8], fused[:, :8], pos, table, k=fused[:, 8:10], k_out=fused[:, 8:10])   # in place
    assert torch.equal(fused[:, :8], qo) and torch.equal(fused[:, 8:10], ko)
    assert torch.equal(fused[:, 10:], want[:, 10:])
    # heads outermost, rows on a 2-byte boundary only, odd token stride
    flat = torch.zeros(8 * 11 * 131 + 1, dtype=torch.bfloat16, device="cuda")[1:]
    odd = flat.view(8, 11, 131)[..., :128].transpose(0, 1)
    odd.copy_(want[:, :8])
    out = torch.zeros_like(flat).view(8, 11, 131)[..., :128].transpose(0, 1)
    R.reskv_rope(odd, out, pos, table)
    assert torch.equal(out, qo)
    odd_in = torch.as_strided(torch.zeros(3 + 11 * 1024, dtype=torch.bfloat16, device="cuda"), (11, 8, 128), (1024, 128, 1), 3)
    odd_in.copy_(want[:, :8])
    R.reskv_rope(odd_in, odd_in, pos, table)
    assert torch.equal(odd_in, qo)


def test_table_on_an_eight_byte_boundary():
    rng = np.random.default_rng(9)
    tab = po.table(30, po.frequencies(64)).astype(np.float32)
    held = torch.zeros(tab.size + 2, device="cuda")
    held[2:] = torch.from_numpy(tab).cuda().flatten()
    x = torch.from_numpy(rows(rng, (20, 3), 64)).bfloat16().cuda()
    pos = torch.arange(20, dtype=torch.int32, device="cuda") + 10
    for inter in (False, True):
        a, b = torch.empty_like(x), torch.empty_like(x)
        R.reskv_rope(x, a, pos, held[2:].view(30, 32, 2), interleaved=inter)
        R.reskv_rope(x, b, pos, torch.from_numpy(tab).cuda(), interleaved=inter)
        assert torch.equal(a, b)


def test_padding_and_positions_outside_the_table():
    rng = np.random.default_rng(2)
    table = torch.from_numpy(po.table(8, po.frequencies(64)).astype(np.float32)).cuda()
    x = torch.from_numpy(rows(rng, (4, 2), 64)).cuda()
    y = torch.empty_like(x)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    R.reskv_rope(x, y, torch.tensor([-1, 7, 8, 0], dtype=torch.int32, device="cuda"), table, status=status)
    assert torch.equal(y[0], x[0]) and torch.equal(y[2], x[2]) and torch.equal(y[3], x[3])
    assert not torch.equal(y[1], x[1]) and int(status) == 2
    status.zero_()
    R.reskv_rope(x, y, torch.tensor([-1, 7, -5, 0], dtype=torch.int32, device="cuda"), table, status=status)
    assert int(status) == 0
    R.reskv_rope(x[:0], y[:0], torch.empty(0, dtype=torch.int32, device="cuda"), table)


SCALINGS = [("none", R.RESKV_ROPE_NONE, 1.0), ("linear", R.RESKV_ROPE_LINEAR, 4.0), ("base", R.RESKV_ROPE_BASE, 8.0),
            ("wavelength", R.RESKV_ROPE_WAVELENGTH, 8.0), ("yarn", R.RESKV_ROPE_YARN, 16.0)]


@pytest.mark.parametrize("rot", [2, 64, 128, 512])
@pytest.mark.parametrize("name,kind,factor", SCALINGS)
def test_table_matches_fp64(rot, name, kind, factor):
    if rot == 2 and name == "base":
        pytest.skip("needs rot_dim >= 4")
    n = 70000 if rot == 128 else 300
    t = R.reskv_rope_table(R.reskv_rope_config_default(rot_dim=rot, scaling=kind, factor=factor), n).double().cpu().numpy()
    m = 0.1 * np.log(factor) + 1 if name == "yarn" else 1.0
    ref = po.table(n, po.frequencies(rot, scaling=name, factor=factor), m)
    # one rounding to fp32, and the angle's fp64 rounding (pow and product: a few units of 2^-53 of 7e4)
    assert np.abs(t - ref).max() <= 2.0 ** -24 * m + 2.0 ** -32
    t2 = R.reskv_rope_table(R.reskv_rope_config_default(rot_dim=rot, scaling=kind, factor=factor, magnitude=0.5), 5)
    ref2 = po.table(5, po.frequencies(rot, scaling=name, factor=factor), 0.5)
    assert np.abs(t2.double().cpu().numpy() - ref2).max() <= 2.0 ** -24
