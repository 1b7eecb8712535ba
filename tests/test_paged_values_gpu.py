"""Unusual held values in attention over the paged cache: NaN whose weight vanishes."""
import pytest
import torch

from paged_cases import DT
from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


def filled(k, v, page=64):
    """A cache of one sequence with the fp32 rows k, v [n, kv, 128], in pages in reverse order."""
    n, kv, d = k.shape
    pages = -(-n // page)
    table = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device="cuda")[None].contiguous()
    cache = R.PagedKV(R.reskv_paged_pages(pages, kv, page, d, 32), table, page, kv, d, 32)
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
