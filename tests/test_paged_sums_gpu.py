"""Long sums of the few-row kernel against 64 bits."""
import pytest
import torch

from paged_cases import DT
from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,group", [(128, 32), (128, 128), (64, 64)])
@pytest.mark.parametrize("dtype,per", [("bf16", 4), ("f16", 4), ("bf16", 1)])      # per 1, one token: four rows
def test_fp32_outputs_of_long_pieces(d, group, dtype, per):
    """So many units that a warp takes hundreds of tiles of one.

    Tolerance: the sum of w s n (codes n of 7.5 on average, scales s) is formed by one product per tile and plane of
    the weights, each cut off by at most 2^-23 of a sum of 16 tiles, half of that on average, while the outputs are
    rms(o): 2 2^-23 (8 16 7.5 s) / (16 rms(o)) of the output = 2^-23 120 s / rms(o), a worst case in which all cuts
    fall one way by their most.  Fp32 logits, weights and minima add less than 2^-16."""
    n, kv, B, new = 8192, 8, (2 if per > 1 else 300), (128 if per > 1 else 1)
    g = torch.Generator(device="cuda").manual_seed(d + group)
    per_seq = n // 64
    share = B if per > 1 else 3                        # sequences of their own; the others read the same pages
    pages = R.reskv_paged_pages(share * per_seq, kv, 64, d, group)
    table = torch.randperm(share * per_seq, generator=g, device="cuda").to(torch.int32).view(share, per_seq)
    own = R.PagedKV(pages, table, 64, kv, d, group)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    for b in range(share):
        k, v = (torch.randn((n, kv, d), generator=g, device="cuda") for _ in range(2))
        R.reskv_paged_append(own, k, v, torch.full_like(pos, b), pos)
    cache = R.PagedKV(pages, table.repeat(B // share, 1).contiguous(), 64, kv, d, group)
    kk, vv = (torch.empty((share, kv, n, d), device="cuda") for _ in range(2))
    R.reskv_paged_gather(own, torch.full((share,), n, dtype=torch.int32, device="cuda"), kk, vv)
    q = torch.randn((B * new, kv * per, d), generator=g, device="cuda").to(DT[dtype])
    o = torch.full(q.shape, float("nan"), device="cuda")
    begins = (torch.arange(B + 1, device="cuda") * new).to(torch.int32)
    R.reskv_paged_attn(cache, q, torch.full((B,), n, dtype=torch.int32, device="cuda"), o, q_begin=begins)
    cache.check_status()
    see = torch.arange(n, device="cuda") <= (n - new + torch.arange(new, device="cuda"))[:, None]
    off = size = 0.0
    for b in range(B):
        qq = q[b * new:(b + 1) * new].double().view(new, kv, per, d)
        x = torch.einsum("nkad,ktd->kant", qq, kk[b % share].double()) * d ** -0.5
        w = torch.softmax(x.masked_fill(~see, -float("inf")), -1)
        want = torch.einsum("kant,ktd->nkad", w, vv[b % share].double()).reshape(new, kv * per, d)
        off += (o[b * new:(b + 1) * new].double() - want).square().sum().item()
        size += want.square().sum().item()
    rms = (size / o.numel()) ** 0.5
    y = vv.unflatten(-1, (-1, group))
    s = ((y.amax(-1) - y.amin(-1)) / 15).mean().item()
    assert (off / size) ** 0.5 <= 2.0 ** -23 * 120 * s / rms + 2.0 ** -16, ((off / size) ** 0.5, s, rms)
