"""Writing and reading the paged 4-bit cache: held bytes and read values equal the
definition's bit for bit."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paged_cases import DT, as_type, paged, rows
from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


def expect(pages, table, page, d, group, k, v, seqs, positions, tab, interleaved):
    """Pages after holding fp32 rows k, v [T, kv, d]."""
    pages = pages.copy()
    for i, (b, p) in enumerate(zip(seqs, positions)):
        if p < 0:
            continue
        kk = k[i:i + 1] if tab is None else po.rotate(k[i:i + 1], tab[p][None], interleaved)
        for which, x in ((0, kk[0]), (1, v[i])):
            n, s, m = po.hold(x, group)
            for h in range(x.shape[0]):
                po.put_row(pages[table[b, p // page]], h, p % page, d, group, which, n[h], s[h], m[h])
    return pages


def append(rng, kv, d, group, page, dtype, counts, first, interleaved=False, rot=None, k=None, v=None):
    """Append counts[b] tokens from position first[b] of every sequence b in shuffled order; check the pages."""
    cap = [f + c for f, c in zip(first, counts)]
    kvc, _, pages, table = paged(rng, [0] * len(counts), kv, d, group, page, extra_pages=sum(-(-c // page) for c in cap) + 2,
                                 table_pages=max(-(-c // page) for c in cap))
    order = rng.permutation(len(pages))
    at = 0
    for b, c in enumerate(cap):
        table[b, :-(-c // page)] = order[at:at + -(-c // page)]
        at += -(-c // page)
    kvc.page_table.copy_(torch.from_numpy(table))
    seqs = np.repeat(np.arange(len(counts)), counts).astype(np.int32)
    pos = np.concatenate([f + np.arange(c) for f, c in zip(first, counts)]).astype(np.int32)
    mix = rng.permutation(len(seqs))
    seqs, pos = seqs[mix], pos[mix]
    pos = np.where(rng.random(len(pos)) < 0.1, -1, pos).astype(np.int32)
    k = rows(rng, (len(seqs), kv), d) if k is None else k
    v = rows(rng, (len(seqs), kv), d) if v is None else v
    kt, k64 = as_type(k, dtype)
    vt, v64 = as_type(v, dtype)
    tab = None if rot is None else po.table(max(cap) + 1, po.frequencies(rot)).astype(np.float32)
    R.reskv_paged_append(kvc, kt, vt, torch.from_numpy(seqs).cuda(), torch.from_numpy(pos).cuda(),
                         table=None if tab is None else torch.from_numpy(tab).cuda(), interleaved=interleaved)
    want = expect(pages, table, page, d, group, k64.astype(np.float32), v64.astype(np.float32), seqs, pos, tab, interleaved)
    kvc.check_status()
    np.testing.assert_array_equal(kvc.pages.cpu().numpy(), want)


@pytest.mark.parametrize("d,group", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("page,counts,first", [(16, (1,), (0,)), (64, (1, 1, 1), (63, 64, 5)), (32, (35, 1, 20), (3, 31, 0))])
def test_held_bytes(d, group, dtype, page, counts, first):
    rng = np.random.default_rng(d + group + page)
    append(rng, 3, d, group, page, dtype, counts, first, rot=d)
    append(rng, 2, d, group, page, dtype, counts, first, rot=d // 2, interleaved=True)


@pytest.mark.parametrize("rot,interleaved", [(2, False), (6, False), (10, True), (24, False), (64, True), (128, True), (None, False)])
def test_held_bytes_partial_rotation(rot, interleaved):
    append(np.random.default_rng(3), 1, 128, 32, 16, "bf16", (9, 4), (2, 0), rot=rot, interleaved=interleaved)


def test_held_bytes_of_unusual_groups():
    """Constant groups, zeros, subnormals, huge values, infinities and NaN, exact ties of the codes."""
    rng = np.random.default_rng(4)
    x = rows(rng, (12, 2), 128)
    x[0] = 0
    x[1] = 3.25
    x[2] = rng.standard_normal((2, 128)) * 1e-39
    x[3] = rng.standard_normal((2, 128)) * 1e-37
    x[4] = rng.standard_normal((2, 128)) * 1e38
    x[5, 0, 7], x[5, 1, 40], x[6, 0, 100] = np.inf, -np.inf, np.nan
    x[7, 0, ::2], x[7, 0, 1::2] = 3.3e38, -3.3e38
    x[8] = np.tile(np.arange(32) / 2 - 0.5, 4)                    # scale 1: codes at every half
    x[9] = np.tile(np.arange(32) * 7.5 / 15 + 100, 4)             # far from zero
    x[10] = -0.0
    x[11] = 5 + rng.standard_normal((2, 128)) * 1e-3
    for dtype in ("f32", "bf16"):
        append(rng, 2, 128, 32, 16, dtype, (12,), (0,), k=x, v=x[:, ::-1].copy())
        append(rng, 2, 128, 128, 16, dtype, (12,), (0,), k=x, v=x[:, ::-1].copy())


def test_queries_turn_in_the_same_call_and_strides():
    rng = np.random.default_rng(6)
    T, kv, heads, d = 13, 2, 8, 128
    kvc, _, pages, table = paged(rng, [0], kv, d, 32, 16, extra_pages=3, table_pages=2)
    kvc.page_table.copy_(torch.tensor([[2, 0]], dtype=torch.int32))
    tab = torch.from_numpy(po.table(40, po.frequencies(d)).astype(np.float32)).cuda()
    fused = torch.from_numpy(rows(rng, (T, heads + 2 * kv), d)).bfloat16().cuda()
    q, k, v = fused[:, :heads], fused[:, heads:heads + kv], fused[:, heads + kv:]
    pos = torch.arange(T, dtype=torch.int32, device="cuda") + 4
    pos[5] = -1
    seqs = torch.zeros(T, dtype=torch.int32, device="cuda")
    qo, ref = torch.empty((T, heads, d), dtype=torch.bfloat16, device="cuda"), torch.empty((T, heads, d), dtype=torch.bfloat16, device="cuda")
    R.reskv_rope(q, ref, pos, tab)
    R.reskv_paged_append(kvc, k, v, seqs, pos, table=tab, q=q, q_out=qo)
    assert torch.equal(qo, ref)
    a = kvc.pages.clone()
    kvc.pages.fill_(0xFF)
    odd = [torch.as_strided(torch.zeros(1 + T * kv * d, dtype=torch.bfloat16, device="cuda"), (T, kv, d), (kv * d, d, 1), 1) for _ in range(2)]
    odd[0].copy_(k)
    odd[1].copy_(v)
    R.reskv_paged_append(kvc, odd[0], odd[1], seqs, pos, table=tab)         # rows on a 2-byte boundary
    assert torch.equal(a, kvc.pages)
    fused_q = fused.clone()
    R.reskv_paged_append(kvc, fused_q[:, heads:heads + kv], fused_q[:, heads + kv:], seqs, pos, table=tab,
                         q=fused_q[:, :heads], q_out=fused_q[:, :heads])   # in place
    assert torch.equal(fused_q[:, :heads], ref) and torch.equal(fused_q[:, heads:], fused[:, heads:])
    assert torch.equal(a, kvc.pages)


def test_faults_are_reported_and_write_nothing():
    rng = np.random.default_rng(8)
    kvc, _, pages, table = paged(rng, [16, 16], 1, 64, 32, 16, table_pages=3)
    tab = torch.from_numpy(po.table(20, po.frequencies(64)).astype(np.float32)).cuda()
    x = torch.ones((1, 1, 64), device="cuda")
    before = kvc.pages.clone()
    for seq, pos in ((2, 0), (-1, 0), (0, 48), (0, 20), (1, 17), (0, 2 ** 31 - 1)):
        R.reskv_paged_append(kvc, x, x, torch.tensor([seq], dtype=torch.int32, device="cuda"),
                             torch.tensor([pos], dtype=torch.int32, device="cuda"), table=tab)
        with pytest.raises(R.ReskvError) as e:
            kvc.check_status()
        assert e.value.status == R.RESKV_ERR_DEVICE_STATUS, (seq, pos)
        assert torch.equal(before, kvc.pages)
    kvc.check_status()
    R.reskv_paged_append(kvc, x[:0], x[:0], torch.empty(0, dtype=torch.int32, device="cuda"),
                         torch.empty(0, dtype=torch.int32, device="cuda"))


def as_out(x, dtype):
    """fp64 held values rounded to fp32, then to the type, as the library does."""
    return torch.from_numpy(x.astype(np.float32)).to(DT[dtype])


@pytest.mark.parametrize("d,group", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gathered_values(d, group, dtype):
    rng = np.random.default_rng(d * group)
    lens = [37, 0, 16, 1]
    kvc, values, _, _ = paged(rng, lens, 3, d, group, 16)
    lt = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for n, starts in ((40, None), (1, [36, 0, 15, 0]), (21, [5, 3, 9, 0]), (3, [-2, 0, 20, 1])):
        want = torch.zeros((2, 4, 3, n, d), dtype=DT[dtype])
        for b in range(4):
            for i in range(n):
                p = (starts[b] if starts else 0) + i
                if 0 <= p < lens[b]:
                    for w in range(2):
                        want[w, b, :, i] = as_out(values[b][w][:, p], dtype)
        st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
        k, v = (torch.full((4, 3, n, d), float("nan"), dtype=DT[dtype], device="cuda") for _ in range(2))
        R.reskv_paged_gather(kvc, lt, k, v, starts=st)
        assert torch.equal(k.cpu(), want[0]) and torch.equal(v.cpu(), want[1])
        # one of the two, [batch, n, kv, d] memory, rows on an element boundary only
        v2 = torch.full((1 + 4 * n * 3 * d,), float("nan"), dtype=DT[dtype], device="cuda")[1:].view(4, n, 3, d).transpose(1, 2)
        R.reskv_paged_gather(kvc, lt, v_out=v2, starts=st)
        assert torch.equal(v2.cpu(), want[1])
    kvc.check_status()


def test_gather_of_a_missing_page():
    kvc, values, _, table = paged(np.random.default_rng(1), [40], 1, 128, 32, 16)
    kvc.page_table[0, 1] = len(kvc.pages)
    k = torch.full((1, 1, 40, 128), float("nan"), device="cuda")
    R.reskv_paged_gather(kvc, torch.tensor([40], dtype=torch.int32, device="cuda"), k)
    assert (k[0, 0, 16:32] == 0).all() and torch.equal(k[0, 0, :16].cpu(), as_out(values[0][0][0, :16], "f32"))
    with pytest.raises(R.ReskvError):
        kvc.check_status()
    # a length past the table: rows beyond it are a fault too, and zero
    k.fill_(float("nan"))
    kvc.page_table[0, 1] = int(table[0, 1])
    big = torch.full((1, 1, 60, 128), float("nan"), device="cuda")
    R.reskv_paged_gather(kvc, torch.tensor([60], dtype=torch.int32, device="cuda"), big)
    assert (big[0, 0, 48:] == 0).all()
    with pytest.raises(R.ReskvError):
        kvc.check_status()


@pytest.mark.parametrize("kv,heads,d,group,rot,interleaved,dtype", [(3, 6, 128, 32, 128, False, "bf16"), (8, 8, 64, 64, 32, True, "f16"),
                                                                    (5, 7, 128, 128, 64, False, "f32")])
def test_a_large_call_equals_small_ones(kv, heads, d, group, rot, interleaved, dtype):
    """Calls large enough to take several heads a thread hold and turn what small calls do."""
    T = 2 * 152 * 8192 // (kv * d // 8) + 37
    g = torch.Generator(device="cuda").manual_seed(kv)
    k, v, q = (torch.randn((T, h, d), generator=g, device="cuda").to(DT[dtype]) for h in (kv, kv, heads))
    tab = R.reskv_rope_table(R.reskv_rope_config_default(rot_dim=rot), T + 9)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") + 9
    seqs = torch.zeros(T, dtype=torch.int32, device="cuda")
    n = -(-(T + 9) // 64)
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32)[None]
    a, b = (R.PagedKV(R.reskv_paged_pages(n, kv, 64, d, group), table, 64, kv, d, group) for _ in range(2))
    qa, qb, qc = (torch.empty_like(q) for _ in range(3))
    R.reskv_paged_append(a, k, v, seqs, pos, table=tab, interleaved=interleaved, q=q, q_out=qa)
    for i in range(0, T, 4096):
        s = slice(i, i + 4096)
        R.reskv_paged_append(b, k[s], v[s], seqs[s], pos[s], table=tab, interleaved=interleaved, q=q[s], q_out=qb[s])
    R.reskv_rope(q, qc, pos, tab, interleaved=interleaved)
    a.check_status()
    assert torch.equal(a.pages, b.pages) and torch.equal(qa, qb) and torch.equal(qa, qc)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotated_rows_equal_rounded_products_and_sums(interleaved):
    """Many fp32 rows: every product and sum of the rotation is rounded on its own, held keys included."""
    T, kv, d = 4096, 2, 128
    g = torch.Generator(device="cuda").manual_seed(11)
    k = torch.randn((T, kv, d), generator=g, device="cuda")
    tab = R.reskv_rope_table(R.reskv_rope_config_default(), T)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    c, s = tab[:, None, :, 0], tab[:, None, :, 1]
    a, b = (k[..., 0::2], k[..., 1::2]) if interleaved else (k[..., :64], k[..., 64:])
    x, y = a * c - b * s, b * c + a * s                                  # one operation a kernel: nothing fused
    want = torch.stack([x, y], -1).flatten(-2) if interleaved else torch.cat([x, y], -1)
    got = torch.empty_like(k)
    R.reskv_rope(k, got, pos, tab, interleaved=interleaved)
    assert torch.equal(got, want)
    pages = [R.reskv_paged_pages(64, kv) for _ in range(2)]
    table = torch.arange(64, dtype=torch.int32, device="cuda")[None]
    seqs = torch.zeros(T, dtype=torch.int32, device="cuda")
    R.reskv_paged_append(R.PagedKV(pages[0], table, 64, kv), k, k, seqs, pos, table=tab, interleaved=interleaved)
    R.reskv_paged_append(R.PagedKV(pages[1], table, 64, kv), want, k, seqs, pos)
    assert torch.equal(pages[0], pages[1])
