"""The workspaces of reskv_paged_attn: the binding's own, kept per stream, and the caller's."""
import numpy as np
import pytest
import torch

from paged_cases import as_type, paged
from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


def state(seed=70, lens=(900, 1, 400)):
    """Long enough for units that are cut between CTAs: the tickets and records are used."""
    rng = np.random.default_rng(seed)
    kv, _, _, _ = paged(rng, lens, 1, 64, 64, 64)
    q, _ = as_type(rng.standard_normal((len(lens), 4, 64)), "bf16")
    lt = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = torch.empty_like(q)
    R.reskv_paged_attn(kv, q, lt, want)
    return kv, q, lt, want


def own(kv, q):
    return torch.zeros(R.reskv_paged_attn_workspace(kv, *q.shape[:2]), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("by_handle", [False, True])
def test_a_captured_call_brings_its_workspace(monkeypatch, by_handle):
    """Without one it is refused, the capture goes on, and no workspace that was never zeroed is kept."""
    monkeypatch.setattr(R, "_workspaces", {})           # torch hands streams out again
    kv, q, lt, want = state()
    out, ws, side = torch.zeros_like(q), own(kv, q), torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        with pytest.raises(ValueError, match="workspace="):
            R.reskv_paged_attn(kv, q, lt, out, stream=side.cuda_stream if by_handle else None)
        assert (q.get_device(), side.cuda_stream) not in R._workspaces
        R.reskv_paged_attn(kv, q, lt, out, workspace=ws)
    for _ in range(2):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    with torch.cuda.stream(side):                      # the stream by itself
        for _ in range(2):
            out.zero_()
            R.reskv_paged_attn(kv, q, lt, out)
            side.synchronize()
            assert torch.equal(out, want)
    # and again in a capture, though the stream now has a workspace
    with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
        with pytest.raises(ValueError, match="workspace="):
            R.reskv_paged_attn(kv, q, lt, out)
        out.zero_()
    kv.check_status()


def test_a_workspace_that_could_not_be_zeroed_is_not_kept(monkeypatch):
    monkeypatch.setattr(R, "_workspaces", {})
    kv, q, lt, want = state()
    side, out = torch.cuda.Stream(), torch.zeros_like(q)
    torch.cuda.synchronize()

    class Refuses:
        def __init__(self, stream):
            self.stream = stream

        def synchronize(self):
            raise RuntimeError("not now")

    current = torch.cuda.current_stream
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Refuses(current(*a)))
    with pytest.raises(RuntimeError, match="not now"):
        R.reskv_paged_attn(kv, q, lt, out, stream=side.cuda_stream)
    monkeypatch.setattr(torch.cuda, "current_stream", current)
    assert not R._workspaces.get((q.get_device(), side.cuda_stream))
    R.reskv_paged_attn(kv, q, lt, out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)


def test_kept_workspaces_are_zeroed_in_place_after_a_wait_that_gave_up(monkeypatch):
    """Every stream's, none dropped: work in flight may be using it."""
    monkeypatch.setattr(R, "_workspaces", {})
    kv, q, lt, want = state()
    side, out = torch.cuda.Stream(), torch.zeros_like(q)
    R.reskv_paged_attn(kv, q, lt, out, stream=side)
    torch.cuda.synchronize()
    kept = [w for held in R._workspaces.values() for w in held]
    assert len(kept) == 2
    at = [w.data_ptr() for w in kept]
    for w in kept:
        w.fill_(0x11)
    kv.status.fill_(1)                                 # what a kernel whose wait gave up reports
    with pytest.raises(R.ReskvError, match="word 1"):
        kv.check_status()
    now = [w for held in R._workspaces.values() for w in held]
    assert [w.data_ptr() for w in now] == at and all((w == 0).all() for w in now)
    for stream in (None, side):
        out.zero_()
        torch.cuda.synchronize()
        R.reskv_paged_attn(kv, q, lt, out, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    for w in kept:
        w.fill_(0x11)
    kv.status.fill_(2)                                 # an index out of range leaves them ready
    with pytest.raises(R.ReskvError, match="word 2"):
        kv.check_status()
    assert all((w == 0x11).all() for w in kept)
    for w in kept:
        w.zero_()


def test_workspaces_that_are_refused():
    """Host memory, rows that do not lie together, too few bytes; any type of enough bytes will do."""
    kv, q, lt, want = state()
    n = own(kv, q).numel()
    out = torch.zeros_like(q)
    for bad in (torch.zeros(n, dtype=torch.uint8), torch.zeros(n, dtype=torch.uint8).pin_memory(),
                torch.zeros((n, 2), dtype=torch.uint8, device="cuda")[:, 0], torch.zeros((2, n), dtype=torch.uint8, device="cuda").t()):
        with pytest.raises(ValueError, match="workspace must be"):
            R.reskv_paged_attn(kv, q, lt, out, workspace=bad)
    for few in (own(kv, q)[:-1], own(kv, q)[16:], torch.zeros(n // 4 - 1, dtype=torch.int32, device="cuda")):
        with pytest.raises(R.ReskvError, match="workspace must be"):
            R.reskv_paged_attn(kv, q, lt, out, workspace=few)
    for good in (own(kv, q), torch.zeros(-(-n // 4), dtype=torch.int32, device="cuda")):
        out.zero_()
        R.reskv_paged_attn(kv, q, lt, out, workspace=good)
        assert torch.equal(out, want)
