"""Windows up to the largest int32, with queries that stand before position 0 beside
queries that see everything: a window that reaches past every position is none."""
import numpy as np
import pytest
import torch

from paged_cases import as_type, paged
from paper_2607_29591_gb300 import reskv as R
from test_paged_attn_gpu import case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,out", [(1, "bf16"), (9, "f32"), (40, "f32"), (40, "bf16"), (200, "bf16")])
def test_windows_past_every_position_are_none(new, out):
    """lens from 0 to more than the query tokens; few rows and blocks of 128 and 256."""
    lens, kv, per, d = [3, 0, 25, 150, 37, 260], 1, 4, 128
    kvc, q, lt, o, lse = case(new, lens, new, kv, per, d, 32, 32, "bf16", out=out)
    for window in (2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 150, 1 << 20, 260):
        got, sums = torch.full_like(o, float("nan")), torch.full_like(lse, float("nan"))
        R.reskv_paged_attn(kvc, q, lt, got, window=window, lse=sums)
        kvc.check_status()
        assert torch.equal(got, o) and torch.equal(sums, lse), window


def test_windows_past_every_position_with_ragged_queries():
    rng = np.random.default_rng(60)
    kvc, _, _, _ = paged(rng, [5, 60, 0], 2, 64, 32, 16)
    q, _ = as_type(rng.standard_normal((55, 4, 64)), "f16")
    begins = torch.tensor([0, 30, 50, 55], dtype=torch.int32, device="cuda")
    lt = torch.tensor([5, 60, 0], dtype=torch.int32, device="cuda")
    outs = []
    for window in (0, 2 ** 31 - 1):
        outs.append(torch.full_like(q, float("nan")))
        R.reskv_paged_attn(kvc, q, lt, outs[-1], q_begin=begins, window=window)
    kvc.check_status()
    assert torch.equal(*outs)


@pytest.mark.parametrize("window", [1, 30, 149, 150, 151])
def test_windows_about_the_lengths(window):
    case(window, [150, 17, 3], 40, 1, 4, 128, 32, 16, "bf16", window=window, out="f32")
    case(window + 1000, [150, 17, 3], 40, 1, 4, 128, 32, 16, "bf16", window=window)
