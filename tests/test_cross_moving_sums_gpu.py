"""Cross attention of many rows whose largest logit keeps growing: the two threads of a row work on
halves of a tile, agree on its largest logit and write their weights over what both have read, so the
halves of an output row and its log-sum-exp hold together only if each waits for the other.  The
same bits call after call, alone and beside other work, and the fp64 values within the bound of
test_cross_gpu.check."""
import pytest
import torch

from oracle import cross_oracle as co
from test_cross_gpu import Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f16")])
@pytest.mark.parametrize("counts,lens,kv,per", [([700, 300], [3000, 2050], 2, 4), ([30], [4000], 1, 4), ([16] * 40, [1500] * 40, 4, 2)])
def test_growing_logits(counts, lens, kv, per, d, dtype):
    c = Case(31, counts, lens, kv, per, d, dtype)
    for b, (_, r, _) in enumerate(c.sequences()):
        grow = torch.linspace(0.2, 3.0, lens[b], device="cuda")[:, None, None]
        c.k[r] = (c.k[r].float() * grow).to(c.k.dtype)
    c.k64 = c.k.double().cpu().numpy()
    scale = d ** -0.5
    o, lse = c.forward()
    refs = [co.attend(c.q64[t], c.k64[r].transpose(1, 0, 2), c.v64[r].transpose(1, 0, 2), scale) for t, r, _ in c.sequences()]
    check(o, lse, refs, d, dtype)
    beside = torch.cuda.Stream()
    x = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for i in range(30):
        if i % 2:
            with torch.cuda.stream(beside):
                x.mul_(1.0)
        again, lse2 = c.forward()
        assert torch.equal(o.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse2)
    torch.cuda.synchronize()
    assert int(c.status) == 0
