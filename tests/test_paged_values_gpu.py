"""Unusual held values in attention over the paged cache: NaN whose weight vanishes, rows
of constants of any size, logits of any size."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paged_cases import DT, HALF_ULP, as_type
from paper_2607_29591_gb300 import reskv as R
from test_paged_attn_gpu import check

pytestmark = pytest.mark.gpu


def filled(k, v, page=64, group=32):
    """A cache of one sequence with the fp32 rows k, v [n, kv, 128], in pages in reverse order."""
    n, kv, d = k.shape
    pages = -(-n // page)
    table = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device="cuda")[None].contiguous()
    cache = R.PagedKV(R.reskv_paged_pages(pages, kv, page, d, group), table, page, kv, d, group)
    R.reskv_paged_append(cache, k, v, torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda"))
    cache.check_status()
    return cache


@pytest.mark.parametrize("n", [600, 4000, 33000])      # joins in a CTA, across CTAs, of more than 32 records
@pytest.mark.parametrize("new,dtype,out", [(1, "bf16", "bf16"), (1, "f16", "f32"), (2, "bf16", "f32"), (20, "bf16", "bf16"), (20, "f16", "f16")])
def test_nan_of_vanishing_weight_reaches_the_output(n, new, dtype, out):
    """Position 3 holds NaN values in dims 32..63 of KV head 0, with logits hundreds below those of the last quarter:
    0 times NaN is NaN, in whichever part of the positions it lies."""
    g = torch.Generator(device="cuda").manual_seed(n)
    k, v = (torch.randn((n, 2, 128), generator=g, device="cuda") for _ in range(2))
    k = 0.01 * k
    k[3 * n // 4:] += 4.0
    v[3, 0, 40] = float("nan")
    cache = filled(k, v)
    q = torch.full((new, 8, 128), 8.0, device="cuda").to(DT[dtype])
    o, lse = torch.zeros((new, 8, 128), dtype=DT[out], device="cuda"), torch.zeros((new, 8), device="cuda")
    R.reskv_paged_attn(cache, q, torch.tensor([n], dtype=torch.int32, device="cuda"), o, lse=lse)
    cache.check_status()
    assert torch.isnan(o[:, :4, 32:64]).all()
    assert torch.isfinite(o[:, :4, :32]).all() and torch.isfinite(o[:, :4, 64:]).all() and torch.isfinite(o[:, 4:]).all()
    assert torch.isfinite(lse).all()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("new,dtype,out", [(1, "bf16", "bf16"), (1, "f16", "f32"), (3, "bf16", "f32"), (20, "bf16", "bf16")])
@pytest.mark.parametrize("c,mix", [(0.0, False), (1.0, False), (-65504.0, False), (1e9, False), (-1e12, False), (1e9, True)])
def test_rows_of_constants(c, mix, new, dtype, out, group):
    """Values without a scale, under logits that rise along the positions; with `mix` beside rows of their size that
    have one, and zeros.  Tolerance as in test_paged_attn_gpu.py, in units of the values."""
    rng = np.random.default_rng(90)
    n = 700
    # logits from about -20 to 20: the reference follows in steps and within them
    q = 0.5 * rng.standard_normal((new, 4, 128)) + 1.0
    k = np.linspace(-1.8, 1.8, n)[:, None, None] + 0.2 * rng.standard_normal((n, 1, 128))
    v = np.full((n, 1, 128), c)
    if mix:
        v[1::3] = c * rng.standard_normal((len(v[1::3]), 1, 128))
        v[2::3] = 0
    k, v = (torch.from_numpy(x.astype(np.float32)).cuda() for x in (k, v))
    cache = filled(k, v, group=group)
    ln = torch.tensor([n], dtype=torch.int32, device="cuda")
    kk, vv = (torch.empty((1, 1, n, 128), device="cuda") for _ in range(2))
    R.reskv_paged_gather(cache, ln, kk, vv)
    qt, q64 = as_type(q, dtype)
    o, lse = torch.full((new, 4, 128), float("nan"), dtype=DT[out], device="cuda"), torch.empty((new, 4), device="cuda")
    R.reskv_paged_attn(cache, qt, ln, o, lse=lse)
    cache.check_status()
    unit = abs(c) or 1.0
    ro, rl, xm, vm = po.attend(q64, kk[0].double().cpu().numpy(), vv[0].double().cpu().numpy(), 4, 128 ** -0.5)
    check(o.double() / unit, lse, [(ro / unit, rl, xm, vm / unit)], 128, out)


@pytest.mark.parametrize("size", [1e5, 1e7, 1e8, 3e8, 1e9, 1e10, 1e12, 1e15, 1e20])
@pytest.mark.parametrize("n,new,dtype,out", [(300, 1, "bf16", "bf16"), (300, 1, "f16", "f32"), (300, 3, "bf16", "f32"), (4000, 1, "bf16", "f32"),
                                             (300, 20, "bf16", "bf16"), (3100, 12, "f16", "f16"), (300, 70, "bf16", "bf16")])
def test_logits_of_any_size(size, n, new, dtype, out):
    """One key's logit is past what fp32 counts in ones, another's as far below: the output is the one's value.  Its
    weight times the group's scale is rounded to 11 bits, times a code at most the row's range, then the output; the log-sum-exp is the logit, 128 products and
    a scaling of fp32 (129 2^-23 of it)."""
    g = torch.Generator(device="cuda").manual_seed(n + new)
    k, v = 0.1 * torch.randn((n, 1, 128), generator=g, device="cuda"), torch.randn((n, 1, 128), generator=g, device="cuda")
    k[n // 3], k[n // 2] = size, -size
    cache = filled(k, v)
    ln = torch.tensor([n], dtype=torch.int32, device="cuda")
    kk, vv = (torch.empty((1, 1, n, 128), device="cuda") for _ in range(2))
    R.reskv_paged_gather(cache, ln, kk, vv)
    q = (1 + 0.1 * torch.rand((new, 4, 128), generator=g, device="cuda")).to(DT[dtype])
    o, lse = torch.full((new, 4, 128), float("nan"), dtype=DT[out], device="cuda"), torch.empty((new, 4), device="cuda")
    R.reskv_paged_attn(cache, q, ln, o, lse=lse)
    cache.check_status()
    win = vv[0, 0, n // 3]
    tol = 2.0 ** -11 * (win.max() - win.min()) + HALF_ULP[out] * win.abs() * 1.01
    assert ((o.float() - win).abs() <= tol).all()
    logit = (q.double() * kk[0, 0, n // 3].double()).sum(-1) * 128 ** -0.5
    assert ((lse.double() - logit).abs() <= 129 * 2.0 ** -23 * logit.abs()).all()


@pytest.mark.parametrize("k_size,v_size", [(1.0, 1e12), (1e12, 1.0), (3e8, 1e30), (1e-14, 1e-14)])
@pytest.mark.parametrize("n,new,window,at", [
    (150, 30, 0, 140),             # a later token of the chunk: the queries before it do not see it
    (150, 30, 10, 125),            # one that leaves the window: the queries after it do not
    (3100, 12, 0, 3095),           # the same with the positions in parts
    (300, 70, 40, 233),            # blocks of 256 rows
])
def test_blocks_beside_a_token_of_another_size(n, new, window, at, k_size, v_size):
    """One token's key and value are far larger (or smaller) than the others': queries that do not see it, in the same
    block of rows, are as exact as ever.  Tolerance as in test_paged_attn_gpu.py, by what each query sees."""
    rng = np.random.default_rng(91)
    k, v = rng.standard_normal((n, 1, 128)), rng.standard_normal((n, 1, 128))
    k[at] *= k_size
    v[at] *= v_size
    k, v = (torch.from_numpy(x.astype(np.float32)).cuda() for x in (k, v))
    cache = filled(k, v)
    ln = torch.tensor([n], dtype=torch.int32, device="cuda")
    kk, vv = (torch.empty((1, 1, n, 128), device="cuda") for _ in range(2))
    R.reskv_paged_gather(cache, ln, kk, vv)
    q, q64 = as_type(rng.standard_normal((new, 4, 128)), "bf16")
    o, lse = torch.full_like(q, float("nan")), torch.empty((new, 4), device="cuda")
    R.reskv_paged_attn(cache, q, ln, o, lse=lse, window=window)
    cache.check_status()
    ref = po.attend(q64, kk[0].double().cpu().numpy(), vv[0].double().cpu().numpy(), 4, 128 ** -0.5, window)
    check(o, lse, [ref], 128, "bf16")
    again = torch.empty_like(o)
    R.reskv_paged_attn(cache, q, ln, again, window=window)
    assert torch.equal(o, again)
