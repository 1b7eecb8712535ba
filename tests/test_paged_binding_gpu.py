"""The two ways of a small call from torch tensors to the library: plain CUDA tensors go through host C++, anything else
through Python, with the same results and the same refusals."""
import pytest
import torch

from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


class Sub(torch.Tensor):
    """Not a plain tensor: the general path."""


def sub(t):
    return t.as_subclass(Sub)


def state():
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()     # noqa: E731
    table = R.reskv_rope_table(R.reskv_rope_config_default(), 100)
    return r(6, 8, 128), r(6, 2, 128), r(6, 2, 128), table, torch.arange(6, dtype=torch.int32, device="cuda") + 30


def cache():
    return R.PagedKV(R.reskv_paged_pages(4, 2), torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2), 64, 2)


def test_both_ways_agree(monkeypatch):
    q, k, v, table, pos = state()
    cache()                                            # loads the library
    seqs = torch.tensor([0, 0, 0, 1, 1, 1], dtype=torch.int32, device="cuda")
    lens = torch.tensor([40, 40], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    taken = []
    plain = R._bind

    class Watch:
        def __getattr__(self, name):
            def call(*a):
                taken.append((name, getattr(plain, name)(*a)))
                return taken[-1][1]
            return call

    monkeypatch.setattr(R, "_bind", Watch())
    outs = []
    for wrap, stream in ((lambda t: t, None), (lambda t: t, side), (lambda t: t, side.cuda_stream), (sub, None)):
        kv = cache()
        torch.cuda.synchronize()
        qo, ko, q2 = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
        kk, vv = (torch.empty((2, 2, 40, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        R.reskv_rope(wrap(q), qo, pos, table, k=k, k_out=ko, stream=stream)
        R.reskv_paged_append(kv, wrap(k), v, seqs, pos, table=table, q=q, q_out=q2, stream=stream)
        R.reskv_paged_gather(kv, wrap(lens), kk, vv, stream=stream)
        torch.cuda.synchronize()
        kv.check_status()
        outs.append((qo, ko, q2, kk, vv, kv.pages))
    assert [t for t in taken] == [(n, 0) for n in ("rope", "append", "gather")] * 3 + [(n, -1) for n in ("rope", "append", "gather")]
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], o))


def test_refusals_of_device_tensors():
    q, k, v, table, pos = state()
    kv = cache()
    seqs = torch.zeros(6, dtype=torch.int32, device="cuda")
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    kk = torch.empty((2, 2, 8, 128), device="cuda")
    for wrong in (dict(q=q[:5]), dict(q=q.double()), dict(q=q.cpu()), dict(positions=pos.long()), dict(positions=pos[:3]),
                  dict(positions=pos.repeat(2)[::2]), dict(table=table[..., 0]), dict(table=table.double()),
                  dict(k=k), dict(q_out=q.transpose(1, 2).contiguous().transpose(1, 2))):
        a = dict(dict(q=q, q_out=q.clone(), positions=pos, table=table), **wrong)
        with pytest.raises((ValueError, TypeError)):
            R.reskv_rope(**a)
    with pytest.raises(R.ReskvError, match="n_positions|rot_dim|head_dim"):
        R.reskv_rope(q, q.clone(), pos, torch.zeros((10, 65, 2), device="cuda"))
    for wrong in (dict(k=k[:, :1]), dict(v=v[:5]), dict(seqs=seqs.long()), dict(q=q), dict(q=q, q_out=q[:, :4]), dict(v=v[..., :64])):
        with pytest.raises((ValueError, TypeError)):
            R.reskv_paged_append(kv, **dict(dict(k=k, v=v, seqs=seqs, positions=pos), **wrong))
    for a in ((lens.long(), kk, kk), (lens[:1], kk, kk), (lens, kk[:, :1], None), (lens, kk, kk[:, :, :4]), (lens, None, None),
              (lens, kk.double(), None)):
        with pytest.raises((ValueError, TypeError)):
            R.reskv_paged_gather(kv, *a)
    R.reskv_rope(q[:0], q[:0], pos[:0], table)         # nothing to do
    kv.check_status()
