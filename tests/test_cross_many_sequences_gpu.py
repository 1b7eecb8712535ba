"""Packed batches of many sequences: the same bits as each sequence's rows give in a batch that needs no search, gaps
and empty sequences among them, faults wherever they stand, and a time that grows with the batch, not its square."""
import numpy as np
import pytest
import torch

from cross_cases import check_norms
from test_cross_gpu import Case
from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch", [1, 31, 32, 33, 64, 65, 1000, 1025])
@pytest.mark.parametrize("most", [2, 40])
def test_ragged_batches(batch, most):
    rng = np.random.default_rng(batch + most)
    counts, lens = rng.integers(0, most + 1, batch).tolist(), rng.integers(0, 30, batch).tolist()
    c = Case(101, counts, lens, 1, 3 if most == 2 else 2, 64, "bf16", gap=batch % 7)
    c.check()
    check_norms(c)


@pytest.mark.parametrize("n", [1, 20])
def test_one_long_sequence_among_empty_ones(n):
    for at in (0, 17, 599):
        counts, lens = [0] * 600, [1] * 600
        counts[at], lens[at] = 300 * n, 500
        Case(102, counts, lens, 2, 2, 64, "f16").check()


@pytest.mark.parametrize("batch,n", [(5000, 1), (40000, 1), (3000, 20)])
def test_packed_as_equal(batch, n):
    """Equal lengths by begins, and without: the same bits."""
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((batch * m, h, 64), generator=g, device="cuda").half() for m, h in ((n, 4), (8, 2), (8, 2)))
    begin = lambda m: torch.arange(batch + 1, dtype=torch.int32, device="cuda") * m  # noqa: E731
    out = []
    for a in (dict(), dict(q_begin=begin(n), kv_begin=begin(8))):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        o, lse = torch.full_like(q, 7), torch.empty(q.shape[:2], device="cuda")
        grads = [torch.full_like(t, 7) for t in (q, k, v)]
        R.reskv_cross_attn(q, k, v, o, batch=batch, lse=lse, status=status, **a)
        R.reskv_cross_attn_backward(q, k, v, o, lse, q, *grads, batch=batch, status=status, **a)
        assert int(status) == 0
        out.append((o, lse, *grads))
    for a, b in zip(*out):
        assert torch.equal(a, b)


@pytest.mark.parametrize("where", [0, 1, 33, 700, 2999, 3000])
@pytest.mark.parametrize("which", ["q_begin", "kv_begin"])
def test_a_fault_anywhere_is_reported(which, where):
    batch = 3000
    q, k = (torch.randn((batch * m, 2, 64), device="cuda").half() for m in (1, 4))
    a = dict(q_begin=torch.arange(batch + 1, dtype=torch.int32, device="cuda"), kv_begin=torch.arange(batch + 1, dtype=torch.int32, device="cuda") * 4)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    R.reskv_cross_attn(q, k, k, o, batch=batch, lse=lse, status=status, **a)
    assert int(status) == 0
    for bad in (-1, 1 << 30):
        kept = a[which][where].clone()
        a[which][where] = bad
        status.zero_()
        R.reskv_cross_attn(q, k, k, o, batch=batch, lse=lse, status=status, **a)
        assert int(status) == 2
        status.zero_()
        grads = [torch.zeros_like(t) for t in (q, k, k)]
        R.reskv_cross_attn_backward(q, k, k, o, lse, q, *grads, batch=batch, status=status, **a)
        assert int(status) == 2
        a[which][where] = kept


def test_time_grows_with_the_batch():
    """16 times the sequences: 16 times the work, and no more than twice that in time (a search of every sequence
    before took 256 times)."""
    def passed(batch):
        q, k = (torch.randn((batch * m, 4, 64), device="cuda").half() for m in (1, 16))
        begin = [torch.arange(batch + 1, dtype=torch.int32, device="cuda") * m for m in (1, 16)]
        o = torch.empty_like(q)
        call = lambda: R.reskv_cross_attn(q, k, k, o, batch=batch, q_begin=begin[0], kv_begin=begin[1])  # noqa: E731
        times = []
        for _ in range(7):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            call()
            a.record()
            call()
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    assert passed(32768) < 32 * passed(2048)
