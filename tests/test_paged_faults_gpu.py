"""Queries beside the faults of an append: nothing is held, and the queries are what
reskv_rope makes of the positions, in the keys' launch as in one of their own."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paged_cases import paged, rows
from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("apart", [False, True])
def test_queries_beside_faults(apart):
    """apart: queries of another type than the keys, turned in a launch of their own."""
    rng = np.random.default_rng(80)
    kv, _, _, table = paged(rng, [16, 16], 1, 64, 32, 16, table_pages=3)
    tab = torch.from_numpy(po.table(20, po.frequencies(64)).astype(np.float32)).cuda()
    # a sequence outside the table (two), a position past its pages, one past n_positions, an entry that
    # names no page, padding, and a token that is held
    at = [(2, 3), (-1, 0), (0, 48), (0, 20), (1, 17), (0, -1), (1, 5)]
    seqs, pos = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in zip(*at))
    k = torch.from_numpy(rows(rng, (len(at), 1), 64)).bfloat16().cuda()
    q = torch.from_numpy(rows(rng, (len(at), 4), 64)).cuda().to(torch.float32 if apart else torch.bfloat16)
    q_out, want = torch.full_like(q, float("nan")), torch.full_like(q, float("nan"))
    one = kv.pages.clone()
    R.reskv_paged_append(kv, k, k, seqs, pos, table=tab, q=q, q_out=q_out)
    with pytest.raises(R.ReskvError, match="word 2"):
        kv.check_status()
    R.reskv_rope(q, want, pos, tab)
    assert torch.equal(q_out, want)
    for i in (2, 3, 5):                                # 48, 20 and -1: outside the table of rotations
        assert torch.equal(q_out[i], q[i])
    assert not torch.equal(q_out[0], q[0]) and not torch.equal(q_out[4], q[4])
    # pages: the one token that is held, and nothing else
    held = kv.pages.clone()
    kv.pages.copy_(one)
    R.reskv_paged_append(kv, k[6:], k[6:], seqs[6:], pos[6:], table=tab)
    kv.check_status()
    assert torch.equal(kv.pages, held) and not torch.equal(held, one)
