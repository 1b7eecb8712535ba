"""A refused attention call makes no workspace, and the next call is as if it had not been."""
import numpy as np
import pytest
import torch

from paged_cases import paged
from paper_2607_29591_gb300 import reskv as R
from test_cross_gpu import Case

pytestmark = pytest.mark.gpu


def test_refused_calls_make_no_workspace():
    kv, _, _, _ = paged(np.random.default_rng(0), [40, 20], 2, 128, 32, 16)
    prefix, _, _, _ = paged(np.random.default_rng(1), [30], 2, 128, 32, 16)
    q, lens, one = torch.randn((2, 4, 128), device="cuda").bfloat16(), torch.tensor([40, 20], dtype=torch.int32, device="cuda"), \
        torch.tensor([30], dtype=torch.int32, device="cuda")
    o, short = torch.zeros_like(q), torch.zeros((1, 4), device="cuda")
    c = Case(91, [3, 4], [20, 30], 1, 2, 64, "bf16")
    good = c.backward(*c.forward())
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        before = dict(R._workspaces)
        for call in (lambda: R.reskv_paged_attn(kv, q, lens, o, lse=short), lambda: R.reskv_paged_attn(kv, q, lens[:1], o),
                     lambda: R.reskv_paged_attn(kv, q, lens, o[:1]), lambda: R.reskv_paged_attn(kv, q, lens, o.to(torch.int8)),
                     lambda: R.reskv_paged_attn_shared(kv, prefix, q, lens, one, o, lse=short),
                     lambda: R.reskv_paged_attn_shared(kv, prefix, q, lens, lens, o),
                     lambda: R.reskv_paged_attn_shared(kv, prefix, q, lens, one, o, seq_begin=one),
                     lambda: c.backward(c.q, torch.zeros((1, 2), device="cuda")), lambda: c.backward(c.q[:3], torch.zeros(c.q.shape[:2], device="cuda"))):
            with pytest.raises(ValueError):
                call()
        assert dict(R._workspaces) == before
        for a, b in zip(good, c.backward(*c.forward())):
            assert torch.equal(a, b)
        R.reskv_paged_attn(kv, q, lens, o)
        R.reskv_paged_attn_shared(kv, prefix, q, lens, one, o)
        kv.check_status()
    assert len(R._workspaces) == len(before) + 1
