"""Appending many tokens of any number of KV heads: what is held, and that a call's work
goes by its rows."""
import pytest
import torch

from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


def tokens(T, kv, d=128, group=32):
    g = torch.Generator(device="cuda").manual_seed(T + kv)
    k, v = (torch.randn((T, kv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    n = -(-T // 64)
    cache = R.PagedKV(R.reskv_paged_pages(n, kv, 64, d, group), torch.arange(n, dtype=torch.int32, device="cuda")[None], 64, kv, d, group)
    return cache, k, v, torch.zeros(T, dtype=torch.int32, device="cuda"), torch.arange(T, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kv", [1, 2, 3, 4, 6, 7, 9, 11, 17])
def test_heads_of_a_large_call(kv):
    """Each head as by itself, in a small call's way."""
    T = 152 * 8192 // (16 * kv) + 41
    cache, k, v, seqs, pos = tokens(T, kv)
    tab = R.reskv_rope_table(R.reskv_rope_config_default(), T)
    R.reskv_paged_append(cache, k, v, seqs, pos, table=tab)
    n = len(cache.pages)
    for h in range(kv):
        one = R.PagedKV(R.reskv_paged_pages(n, 1), cache.page_table, 64, 1)
        for i in range(0, T, 8192):
            s = slice(i, i + 8192)
            R.reskv_paged_append(one, k[s, h:h + 1], v[s, h:h + 1], seqs[s], pos[s], table=tab)
        assert torch.equal(one.pages[:, 0], cache.pages[:, h]), h
    cache.check_status()


def microseconds(call, times=15):
    for _ in range(3):
        call()
    t = []
    for _ in range(times):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        t.append(a.elapsed_time(b) * 1e3)
    return sorted(t)[times // 2]


def test_work_goes_by_the_rows():
    """2^18 rows (65 us of work that instructions bound) of 1, 2 and 4 heads against the same of 8: twice the time is
    allowed, what a thread's eight heads of which one is real would take is 4 to 8 times."""
    def time(kv):
        cache, k, v, seqs, pos = tokens((1 << 18) // kv, kv)
        return microseconds(lambda: R.reskv_paged_append(cache, k, v, seqs, pos))

    base = time(8)
    for kv in (1, 2, 4):
        assert time(kv) <= 2 * base, kv
