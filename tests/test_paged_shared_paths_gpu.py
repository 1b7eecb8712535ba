"""Attention with a shared prefix in forms and sizes of their own: more sequences and groups than one launch holds,
negative scales, tables far wider than what they hold, logits of any size.  Tolerance as in test_paged_shared_gpu."""
import numpy as np
import pytest
import torch

from oracle import cross_oracle as co
from paged_cases import DT, HALF_ULP, as_type, paged
from paper_2607_29591_gb300 import reskv as R
from test_paged_shared_gpu import case

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,out", [("bf16", None), ("f16", "f32")])
@pytest.mark.parametrize("groups,members", [(20, 55), (300, 3), (1023, 1)])
def test_more_sequences_than_a_launch_holds(groups, members, dtype, out):
    lens = [1 + i % 19 for i in range(groups * members)]
    case(31, [(7 * g) % 40 for g in range(groups)], lens, [members] * groups, 1, kv=1, per=2, d=64, page=16, dtype=dtype, out=out)


def test_ragged_groups_of_many_sequences():
    rng = np.random.default_rng(0)
    members = rng.multinomial(1100, [0.2] * 5).tolist()
    counts = rng.integers(0, 3, 1100).tolist()
    case(32, [40, 0, 17, 90, 3], [3 + i % 9 for i in range(1100)], members, None, kv=1, per=2, d=64, page=16, counts=counts)


@pytest.mark.parametrize("batch,new", [(3, 1), (40, 1), (9, 5)])
@pytest.mark.parametrize("dtype,out", [("bf16", None), ("f16", None), ("bf16", "f32")])
def test_negative_scales(batch, new, dtype, out):
    case(33, [150], [new + 5 * i % 60 for i in range(batch)], [batch], new, dtype=dtype, out=out, scale=-0.07)


@pytest.mark.parametrize("batch,new", [(3, 1), (40, 1), (64, 1), (9, 5)])
@pytest.mark.parametrize("own_room,prefix_room", [(400, 1), (1, 4000), (400, 4000)])
def test_tables_wider_than_what_they_hold(batch, new, own_room, prefix_room):
    """The same call with tables of many more pages, whose entries are out of range: fp64's values, and no fault."""
    rng = np.random.default_rng(34)
    prefix, _, _, _ = paged(rng, [500], 2, 128, 32, 16)
    own, _, _, _ = paged(rng, [40] * batch, 2, 128, 32, 16)
    q, _ = as_type(rng.standard_normal((batch * new, 8, 128)), "bf16")
    lens, plens = ints([new + i % 30 for i in range(batch)]), ints([500])
    want, o = torch.empty(q.shape, device="cuda"), torch.empty_like(q)
    R.reskv_paged_attn_shared(own, prefix, q, lens, plens, want)

    def wide(kv, room):
        table = torch.full((kv.batch, kv.table_pages * room), -9, dtype=torch.int32, device="cuda")
        table[:, :kv.table_pages] = kv.page_table
        return R.PagedKV(kv.pages, table, 16, 2, 128, 32)

    a, b = wide(own, own_room), wide(prefix, prefix_room)
    for _ in range(3):
        R.reskv_paged_attn_shared(a, b, q, lens, plens, o)
        a.check_status()
        b.check_status()
        # weights of 11 bits, of held values 11 bits, and half a step of bf16; values within 40, their mean far below
        top = float(want.abs().max())
        assert float((o.float() - want).abs().max()) <= 2.0 ** -9 * top + 40 * (2.0 ** -11 + 2.0 ** -11)


@pytest.mark.parametrize("size", [1e5, 1e7, 1e8, 3e8, 1e9, 1e12, 1e20])
@pytest.mark.parametrize("batch", [3, 40, 64])
@pytest.mark.parametrize("where", ["prefix", "own"])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32")])
def test_logits_of_any_size(dtype, out, where, batch, size):
    """One key's logit is past all others: the output is its value, held in 4 bits.  A value is 11 bits of itself and its group's
    minimum, the weight 11 bits, then the output's half step."""
    rng = np.random.default_rng(35)
    n, kv, d = 300, 1, 128
    prefix, _, _, _ = paged(rng, [0], kv, d, 32, 16, extra_pages=20, table_pages=19)
    prefix.page_table.copy_(torch.arange(19, dtype=torch.int32)[None])
    own, _, _, _ = paged(rng, [0] * batch, kv, d, 32, 16, extra_pages=batch, table_pages=1)
    own.page_table.copy_(torch.arange(batch, dtype=torch.int32)[:, None])
    k, v = 0.1 * rng.standard_normal((n, kv, d)), rng.standard_normal((n, kv, d))
    ko, vo = 0.1 * rng.standard_normal((batch, kv, d)), rng.standard_normal((batch, kv, d))
    k[n // 2] = -size
    (k if where == "prefix" else ko)[n // 3 if where == "prefix" else slice(None)] = size
    f32 = lambda x: torch.from_numpy(x.astype(np.float32)).cuda()  # noqa: E731
    R.reskv_paged_append(prefix, f32(k), f32(v), ints(np.zeros(n)), ints(np.arange(n)))
    R.reskv_paged_append(own, f32(ko), f32(vo), ints(np.arange(batch)), ints(np.zeros(batch)))
    held = [torch.empty((1, kv, n, d), device="cuda") for _ in range(2)]
    mine = [torch.empty((batch, kv, 1, d), device="cuda") for _ in range(2)]
    R.reskv_paged_gather(prefix, ints([n]), *held)
    R.reskv_paged_gather(own, ints(np.ones(batch)), *mine)
    q = (1 + 0.1 * torch.rand((batch, 2, d), device="cuda")).to(DT[dtype])
    o, lse = torch.empty(q.shape, dtype=DT[out], device="cuda"), torch.empty(q.shape[:2], device="cuda")
    R.reskv_paged_attn_shared(own, prefix, q, ints(np.ones(batch)), ints([n]), o, lse=lse)
    own.check_status()
    prefix.check_status()
    win = held[1][0, :, n // 3].expand(batch, d) if where == "prefix" else mine[1][:, 0, 0]
    key = held[0][0, :, n // 3].expand(batch, d) if where == "prefix" else mine[0][:, 0, 0]
    win = win[:, None]
    tol = (2.0 ** -11 + 2.0 ** -10) * win.abs().amax(-1, keepdim=True) * 2 + HALF_ULP[out] * win.abs() * 1.01
    assert ((o.float() - win).abs() <= tol).all()
    logit = (q.double() * key[:, None].double()).sum(-1) * d ** -0.5
    assert ((lse.double() - logit).abs() <= 132 * 2.0 ** -23 * logit.abs()).all()


@pytest.mark.parametrize("batch", [3, 40])
def test_a_prefix_of_all_positions_that_a_table_may_have(batch):
    """2^31 - 16 positions, one page again and again: fp64's attention over that page.  A part's sums grow by a tile of 64
    positions at a time, 2^25 tiles over some 150 parts, each sum off by 2^-23 of itself at most: 2.7 % in all."""
    rng = np.random.default_rng(36)
    many = (1 << 27) - 1
    one, held, _, _ = paged(rng, [16], 1, 64, 32, 16, extra_pages=0)
    prefix = R.PagedKV(one.pages, torch.zeros((1, many), dtype=torch.int32, device="cuda"), 16, 1, 64, 32)
    own, _, _, _ = paged(rng, [1] * batch, 1, 64, 32, 16)
    q, q64 = as_type(rng.standard_normal((batch, 2, 64)) / 4, "bf16")
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    R.reskv_paged_attn_shared(own, prefix, q, ints([1] * batch), ints([16 * many]), o, lse=lse)
    own.check_status()
    prefix.check_status()
    k, v = held[0]
    ro, rl, _, vm = co.attend(q64, k, v, 64 ** -0.5)
    assert (np.abs(o.double().cpu().numpy() - ro) <= 0.06 * vm[..., None]).all()
    assert (np.abs(lse.double().cpu().numpy() - rl - np.log(many)) <= 0.03).all()


@pytest.mark.parametrize("size", [1e1, 1e3, 1e5, 1e6, 1e7, 1e9])
@pytest.mark.parametrize("batch", [1, 3, 7])
def test_equal_keys_of_both_parts_share(batch, size):
    """One key in the prefix and the same as own token, all others far below: one kernel forms both logits, so they are
    equal, and the output is the mean of both values, each off by 11 bits."""
    n, d = 300, 128
    rng = np.random.default_rng(37)
    prefix, _, _, _ = paged(rng, [0], 1, d, 32, 16, extra_pages=20, table_pages=19)
    prefix.page_table.copy_(torch.arange(19, dtype=torch.int32)[None])
    own, _, _, _ = paged(rng, [0] * batch, 1, d, 32, 16, extra_pages=batch, table_pages=1)
    own.page_table.copy_(torch.arange(batch, dtype=torch.int32)[:, None])
    k, v = np.full((n, 1, d), -size / d), rng.standard_normal((n, 1, d))
    ko, vo = np.zeros((batch, 1, d)), rng.standard_normal((batch, 1, d))
    k[100] = ko[:] = (1 + rng.random(d)) * size / d
    f32 = lambda x: torch.from_numpy(x.astype(np.float32)).cuda()  # noqa: E731
    R.reskv_paged_append(prefix, f32(k), f32(v), ints(np.zeros(n)), ints(np.arange(n)))
    R.reskv_paged_append(own, f32(ko), f32(vo), ints(np.arange(batch)), ints(np.zeros(batch)))
    held = [torch.empty((1, 1, n, d), device="cuda") for _ in range(2)]
    mine = [torch.empty((batch, 1, 1, d), device="cuda") for _ in range(2)]
    R.reskv_paged_gather(prefix, ints([n]), *held)
    R.reskv_paged_gather(own, ints(np.ones(batch)), *mine)
    q = (8 + torch.rand((batch, 4, d), device="cuda")).bfloat16()
    o = torch.empty(q.shape, device="cuda")
    R.reskv_paged_attn_shared(own, prefix, q, ints(np.ones(batch)), ints([n]), o)
    a, b = held[1][0, 0, 100], mine[1][:, 0, 0]
    far = float((q.float() @ (held[0][0, 0, 100] - held[0][0, 0, 0])).min()) * d ** -0.5          # the others' logits below
    want, rest = (a + b)[:, None] / 2, n * np.exp(-min(far, 100.0)) * float(held[1].abs().max())
    assert ((o - want).abs() <= 2.0 ** -11 * (a.abs() + b.abs())[:, None] + 2.0 ** -14 + rest).all()
