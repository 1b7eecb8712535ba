"""What attention with a shared prefix refuses, before any launch (no GPU needed; the pointers are never followed)."""
import pytest

from paper_2607_29591_gb300 import build as B
from paper_2607_29591_gb300 import reskv as R

P = 1 << 20                                              # a 256-byte aligned address


@pytest.fixture(scope="module")
def lib():
    B.build()
    return R.load_library()


def heads(data=P, token=4096, head=128, n=32, dtype=R.RESKV_BF16):
    return R.reskv_heads(data, token, head, n, dtype)


def paged(**over):
    f = dict(pages=P, n_pages=10, page_table=P, batch=4, table_pages=5, page_tokens=64, n_kv_heads=8, head_dim=128,
             quant_group=32, status=None)
    f.update(over)
    return R.reskv_paged_kv(**f)


def args(**over):
    f = dict(q=heads(), o=heads(), lens=P, n_tokens=4, workspace=P, workspace_bytes=1 << 34)
    f.update(over)
    return R.reskv_paged_attn_args(**f)


@pytest.mark.parametrize("kv,prefix,a,more,word", [
    ({}, dict(pages=None), {}, {}, "prefix"), ({}, dict(page_tokens=24), {}, {}, "prefix"), (dict(pages=None), dict(batch=1), {}, {}, "pages"),
    ({}, dict(batch=1, head_dim=64), {}, {}, "head_dim"), ({}, dict(batch=1, n_kv_heads=4), {}, {}, ""),
    ({}, dict(batch=1, quant_group=64), {}, {}, "quant_group"), ({}, dict(batch=1, page_tokens=32), {}, {}, "page_tokens"),
    ({}, dict(batch=1), {}, dict(lens=None), "prefix_lens"), ({}, dict(batch=3), {}, dict(seqs=None), "seq_begin"),
    ({}, dict(batch=1), dict(window=5), {}, "window"), ({}, dict(batch=1024), {}, {}, "1024"),
    ({}, dict(batch=1), dict(workspace=None), {}, "workspace"), ({}, dict(batch=1), dict(workspace=P + 16), {}, "workspace"),
    ({}, dict(batch=1), dict(workspace_bytes=4096), {}, "workspace"), ({}, dict(batch=1), dict(n_tokens=5), {}, "multiple of batch"),
    ({}, dict(batch=1), dict(q=heads(dtype=R.RESKV_F32)), {}, "bf16 or fp16"), ({}, dict(batch=1), dict(o=heads(n=8)), {}, "same heads"),
    ({}, dict(batch=1), dict(n_tokens=1 << 20), {}, "2^24"), ({}, dict(batch=1), dict(scale=float("nan")), {}, "scale")])
def test_refusals(lib, kv, prefix, a, more, word):
    m = dict(seqs=P, lens=P)
    m.update(more)
    st = lib.reskv_paged_attn_shared(paged(**kv), paged(**prefix), m["seqs"], m["lens"], args(**a), None)
    assert st == R.RESKV_ERR_INVALID_ARG and word in R.reskv_last_error(), R.reskv_last_error()


def test_workspace_and_nothing_to_do(lib):
    kv, prefix = paged(), paged(batch=1)
    one = lib.reskv_paged_attn_shared_workspace(kv, prefix, args())
    assert one > lib.reskv_paged_attn_workspace(kv, args())          # it may serve reskv_paged_attn, too
    assert lib.reskv_paged_attn_shared_workspace(kv, prefix, args(n_tokens=400)) > one
    for bad in ((None, prefix, args()), (kv, None, args()), (kv, prefix, None), (kv, paged(batch=0), args())):
        assert lib.reskv_paged_attn_shared_workspace(*bad) == 0
    assert lib.reskv_paged_attn_shared(kv, prefix, None, None, args(n_tokens=0), None) == R.RESKV_OK
