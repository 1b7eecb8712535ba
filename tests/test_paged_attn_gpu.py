"""Attention over the paged 4-bit cache against fp64.

Tolerance, from the number formats.  A logit is a sum of d products in fp32,
off by at most d 2^-23 X with X = scale sum |q k| (however the products are
grouped); a weight is then off by a factor of at most 1 + 2 d 2^-23 X, and by
2^-11 where it is rounded to 11 bits for the second product; the sums over
positions add 2^-16.  An output, a mean of values, is off by at most that share
of the largest |v|, then half a unit of its type.
"""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paged_cases import DT, HALF_ULP, as_type, paged, rows
from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


def check(o, lse, refs, d, dtype):
    """o [T, H, d], lse [T, H] against the sequences' attend() results one after another."""
    ro, rl, xm, vm = (np.concatenate([r[i] for r in refs]) for i in range(4))
    got = o.double().cpu().numpy()
    share = 2 * d * 2.0 ** -23 * xm + 2.0 ** -11 + 2.0 ** -16
    tol = (share * vm)[..., None] + HALF_ULP[dtype] * np.abs(ro) * 1.01 + 1e-7
    assert np.isfinite(got).all()
    assert (np.abs(got - ro) <= tol).all(), (np.abs(got - ro) - tol).max()
    if lse is not None:
        gl = lse.double().cpu().numpy()
        assert ((gl == -np.inf) == (rl == -np.inf)).all()
        seen = rl != -np.inf
        assert (np.abs(gl - rl)[seen] <= (d * 2.0 ** -23 * xm + 2.0 ** -12 + 2.0 ** -22 * np.abs(np.where(seen, rl, 0)))[seen]).all()


def attend_all(values, q64, begins, per, scale, window):
    return [po.attend(q64[begins[b]:begins[b + 1]], values[b][0], values[b][1], per, scale, window) for b in range(len(values))]


def case(seed, lens, new, kv, per, d, group, page, dtype, window=0, out=None, ragged=None, scale=None, spread=1.0):
    rng = np.random.default_rng(seed)
    kvc, values, _, _ = paged(rng, lens, kv, d, group, page)
    B, H = len(lens), kv * per
    counts = ragged if ragged is not None else [new] * B
    begins = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    q, q64 = as_type(spread * rng.standard_normal((begins[-1], H, d)), dtype)
    o = torch.full((begins[-1], H, d), float("nan"), dtype=DT[out or dtype], device="cuda")
    lse = torch.full((begins[-1], H), float("nan"), device="cuda")
    lt = torch.tensor(lens, dtype=torch.int32, device="cuda")
    qb = torch.from_numpy(begins).cuda() if ragged is not None else None
    R.reskv_paged_attn(kvc, q, lt, o, q_begin=qb, window=window, lse=lse, scale=scale)
    kvc.check_status()
    refs = attend_all(values, q64, begins, per, scale if scale is not None else d ** -0.5, window)
    check(o, lse, refs, d, out or dtype)
    again = torch.full_like(o, float("nan"))
    R.reskv_paged_attn(kvc, q, lt, again, q_begin=qb, window=window, scale=scale)
    assert torch.equal(o, again)                       # the same bits every time
    return kvc, q, lt, o, lse


@pytest.mark.parametrize("d,group", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("page", [16, 64])
def test_single_tokens(d, group, dtype, page):
    case(1, [1, 0, 15, 16, 17, 64, 65, 200], 1, 2, 4, d, group, page, dtype)


@pytest.mark.parametrize("per", [1, 2, 3, 4, 7, 8, 9, 16, 64])
@pytest.mark.parametrize("new", [1, 3])
def test_head_groups(per, new):
    case(per, [70, 33], new, 2, per, 128, 32, 32, "bf16")


@pytest.mark.parametrize("new", [2, 5, 16, 33, 100, 130])
@pytest.mark.parametrize("d,group,dtype", [(128, 32, "bf16"), (64, 64, "f16")])
def test_several_tokens_are_causal(new, d, group, dtype):
    case(new, [130, 40, 1, 0], new, 2, 4, d, group, 32, dtype)     # some stand before position 0


@pytest.mark.parametrize("window", [1, 2, 16, 17, 50, 1000])
@pytest.mark.parametrize("new", [1, 40])
def test_windows(window, new):
    case(window, [150, 17, 3], new, 1, 4, 128, 32, 16, "bf16", window=window)


def test_ragged_queries():
    case(3, [100, 64, 30, 200, 9], None, 2, 4, 128, 64, 64, "bf16", ragged=[1, 0, 7, 40, 9])
    case(4, [50, 90], None, 2, 2, 64, 32, 16, "f16", ragged=[0, 3])


def test_outputs_in_fp32_and_scale():
    case(5, [300, 77], 2, 2, 4, 128, 32, 64, "bf16", out="f32")
    case(6, [300, 77], 1, 2, 4, 64, 32, 64, "f16", out="f32", scale=0.02)


def test_peaked_and_huge_queries():
    """Logits of hundreds and thousands: the running maximum moves, most weights vanish."""
    case(7, [500], 1, 1, 4, 128, 32, 64, "bf16", spread=30.0)
    case(8, [500], 3, 1, 2, 128, 32, 64, "f16", spread=200.0)
    case(9, [400], 1, 1, 4, 128, 32, 64, "bf16", spread=1e-6)


def test_long_and_many():
    case(10, [3000, 1, 777, 2048], 1, 1, 4, 64, 64, 128, "bf16")
    case(11, list(np.random.default_rng(0).integers(0, 60, 40)), 1, 2, 2, 64, 32, 16, "bf16")
    case(12, list(np.random.default_rng(1).integers(0, 200, 9)), 20, 3, 5, 64, 32, 16, "f16")


def test_values_of_any_size():
    """Scales far from one in keys and values, and very different from token to token."""
    rng = np.random.default_rng(13)
    for kscale, vscale, mixed in ((1e-20, 1e-30, False), (1e-3, 1e30, False), (1.0, 1.0, True), (1e4, 1e-6, True)):
        kvc, _, pages, table = paged(rng, [0], 1, 128, 32, 16, extra_pages=12, table_pages=12)
        kvc.page_table.copy_(torch.arange(12, dtype=torch.int32)[None])
        n = 190
        k, v = rows(rng, (n, 1), 128) * np.float32(kscale), rows(rng, (n, 1), 128) * np.float32(vscale)
        if mixed:
            v *= np.exp(rng.uniform(-9, 9, (n, 1, 1))).astype(np.float32)
        k, v = (torch.from_numpy(x).cuda() for x in (k, v))
        R.reskv_paged_append(kvc, k, v, torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda"))
        ln = torch.tensor([n], dtype=torch.int32, device="cuda")
        kk, vv = (torch.empty((1, 1, n, 128), device="cuda") for _ in range(2))
        R.reskv_paged_gather(kvc, ln, kk, vv)
        q, q64 = as_type(rng.standard_normal((1, 4, 128)) / kscale, "bf16")
        for out in ("f32",):
            o = torch.empty((1, 4, 128), device="cuda")
            lse = torch.empty((1, 4), device="cuda")
            R.reskv_paged_attn(kvc, q, ln, o, lse=lse)
            ref = po.attend(q64, kk[0].double().cpu().numpy(), vv[0].double().cpu().numpy(), 4, 128 ** -0.5)
            if vscale < 1e-6:                      # compare in units of the values
                ref = (ref[0] / vscale, ref[1], ref[2], ref[3] / vscale)
                o = (o.double() / vscale)
            # gathered values carry one fp32 rounding each
            check(o, lse, [ref], 128, "bf16")


def test_what_is_not_seen_does_not_matter():
    """NaN and infinity in every slot past a sequence's end, in its tiles too, and before its window."""
    rng = np.random.default_rng(14)
    lens, kv, d, page = [21, 5], 2, 128, 32
    kvc, values, pages, table = paged(rng, lens, kv, d, 32, page)
    clean = pages.copy()
    q, q64 = as_type(rng.standard_normal((2, 8, d)), "bf16")
    lt = torch.tensor(lens, dtype=torch.int32, device="cuda")
    outs = []
    for fill in (0xFF, 0x00, 0x7F, 0x80):
        p = clean.copy()
        mask = np.full_like(p, 1)
        for b, n in enumerate(lens):                # bytes of held rows stay
            for h in range(kv):
                for t in range(n):
                    z = np.zeros(d, np.uint8)
                    one = np.zeros(d // 32, np.uint16)
                    for w in range(2):
                        keep = np.full((kv, p.shape[2]), 0xFF, np.uint8)
                        po.put_row(keep, h, t % page, d, 32, w, z, one, one)
                        mask[table[b, t // page], h][keep[h] == 0] = 0
        p[mask == 1] = fill
        kvc.pages.copy_(torch.from_numpy(p))
        o = torch.empty((2, 8, d), dtype=torch.bfloat16, device="cuda")
        R.reskv_paged_attn(kvc, q, lt, o)
        outs.append(o)
    assert all(torch.equal(outs[0], o) for o in outs[1:])
    check(outs[0], None, attend_all(values, q64, [0, 1, 2], 4, d ** -0.5, 0), d, "bf16")
    # tokens before the window: NaN scales of the first 10 rows
    kvc.pages.copy_(torch.from_numpy(clean))
    o = torch.empty((2, 8, d), dtype=torch.bfloat16, device="cuda")
    R.reskv_paged_attn(kvc, q, lt, o, window=5)
    p = clean.copy()
    for h in range(kv):
        for t in range(16):
            for w in range(2):
                po.put_row(p[table[0, 0]], h, t, d, 32, w, np.full(d, 15), np.full(4, 0x7FC0), np.full(4, 0x7F80))
    kvc.pages.copy_(torch.from_numpy(p))
    o2 = torch.empty_like(o)
    R.reskv_paged_attn(kvc, q, lt, o2, window=5)
    assert torch.equal(o, o2)
    kvc.check_status()


def test_nan_in_what_is_seen_reaches_the_output():
    kvc, _, pages, table = paged(np.random.default_rng(15), [40, 40], 2, 128, 32, 16)
    page = kvc.pages[int(table[0, 1])].cpu().numpy()
    po.put_row(page, 1, 3, 128, 32, 1, np.zeros(128, np.uint8), np.full(4, 0x7FC0), np.full(4, 0x7FC0))
    kvc.pages[int(table[0, 1])] = torch.from_numpy(page).cuda()
    q = torch.randn((2, 8, 128), dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(q)
    R.reskv_paged_attn(kvc, q, torch.tensor([40, 40], dtype=torch.int32, device="cuda"), o)
    assert torch.isnan(o[0, 4:]).all() and torch.isfinite(o[0, :4]).all() and torch.isfinite(o[1]).all()


def test_strides_and_unaligned_rows():
    kvc, q, lt, o, _ = case(16, [90, 33], 3, 2, 4, 128, 32, 32, "bf16")
    T, H, d = q.shape
    qs = torch.as_strided(torch.zeros(1 + T * H * 200, dtype=q.dtype, device="cuda"), (T, H, d), (200, T * 200, 1), 1)
    os = torch.as_strided(torch.zeros(1 + T * H * 131, dtype=q.dtype, device="cuda"), (T, H, d), (131 * H, 131, 1), 1)
    qs.copy_(q)
    R.reskv_paged_attn(kvc, qs, lt, os)
    assert torch.equal(os, o)
    wide = torch.zeros((T, 3 * H, d), dtype=q.dtype, device="cuda")
    wide[:, H:2 * H] = q
    out = torch.zeros((T, H, 2 * d), dtype=q.dtype, device="cuda")
    R.reskv_paged_attn(kvc, wide[:, H:2 * H], lt, out[..., :d])
    assert torch.equal(out[..., :d], o) and (out[..., d:] == 0).all()


def test_streams_and_graphs():
    kvc, q, lt, o, _ = case(17, [900, 1, 400], 1, 2, 4, 128, 32, 64, "bf16")
    other = torch.cuda.Stream()
    out = torch.zeros_like(o)
    torch.cuda.synchronize()
    R.reskv_paged_attn(kvc, q, lt, out, stream=other)
    other.synchronize()
    assert torch.equal(out, o)
    ws = torch.zeros(R.reskv_paged_attn_workspace(kvc, q.shape[0], q.shape[1]), dtype=torch.uint8, device="cuda")
    out.zero_()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        R.reskv_paged_attn(kvc, q, lt, out, workspace=ws)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o)
    lt.copy_(torch.tensor([899, 1, 400], dtype=torch.int32))       # lengths are read when the kernel runs
    want = torch.empty_like(o)
    R.reskv_paged_attn(kvc, q, lt, want)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and not torch.equal(want[0], o[0])


def test_faults_are_reported():
    rng = np.random.default_rng(18)
    kvc, values, _, table = paged(rng, [64, 64], 1, 128, 32, 16)
    q, q64 = as_type(rng.standard_normal((2, 4, 128)), "bf16")
    o = torch.empty_like(q)
    bad = kvc.page_table.clone()
    for page in (-1, len(kvc.pages), 2 ** 31 - 1):
        kvc.page_table[0, 2] = page
        R.reskv_paged_attn(kvc, q, torch.tensor([64, 64], dtype=torch.int32, device="cuda"), o)
        with pytest.raises(R.ReskvError):
            kvc.check_status()
        check(o[1:], None, attend_all(values[1:], q64[1:], [0, 1], 4, 128 ** -0.5, 0), 128, "bf16")
    kvc.page_table.copy_(bad)
    for n in (-3, 65, 2 ** 31 - 1):                                    # a length outside the table
        R.reskv_paged_attn(kvc, q, torch.tensor([n, 64], dtype=torch.int32, device="cuda"), o)
        with pytest.raises(R.ReskvError):
            kvc.check_status()
        check(o[1:], None, attend_all(values[1:], q64[1:], [0, 1], 4, 128 ** -0.5, 0), 128, "bf16")
    R.reskv_paged_attn(kvc, q, torch.tensor([64, 64], dtype=torch.int32, device="cuda"), o)
    kvc.check_status()
    check(o, None, attend_all(values, q64, [0, 1, 2], 4, 128 ** -0.5, 0), 128, "bf16")


# --- blocks of many query rows (bf16 outputs) ---

@pytest.mark.parametrize("d,group", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64)])
@pytest.mark.parametrize("page,lens,new,per", [(16, [75, 64, 8], 8, 4), (64, [300, 129, 40, 0], 40, 4), (32, [257, 256], 65, 4), (48, [100], 100, 7)])
def test_blocks_of_rows(d, group, page, lens, new, per):
    case(d + page, lens, new, 2, per, d, group, page, "bf16")


@pytest.mark.parametrize("d,group,window", [(128, 32, 0), (64, 64, 0), (128, 128, 700), (128, 32, 90)])
def test_blocks_of_rows_with_their_positions_in_parts(d, group, window):
    """One or two blocks and long contexts: every block's positions go to several CTAs, which may see nothing."""
    case(window + d, [3100, 700], 12, 1, 4, d, group, 64, "bf16", window=window)
    case(window + d + 1, [2100], 70, 1, 4, d, group, 16, "bf16", window=window)


@pytest.mark.parametrize("d,group", [(128, 32), (64, 64)])
def test_blocks_with_fp16_outputs(d, group):
    case(d + 50, [300, 129, 40, 0], 40, 2, 4, d, group, 64, "f16")
    case(d + 51, [3100, 700], 12, 1, 4, d, group, 16, "f16")
    case(d + 52, [257], 65, 2, 4, d, group, 32, "f16", window=100)
    case(d + 53, [500], 20, 1, 4, d, group, 64, "f16", spread=30.0)


def test_blocks_peaked_and_of_any_size():
    """The reference moves by hundreds; values' and keys' magnitudes grow from position to position."""
    case(30, [500], 20, 1, 4, 128, 32, 64, "bf16", spread=30.0)
    case(31, [300], 20, 1, 4, 128, 32, 64, "bf16", spread=1e-6)
    rng = np.random.default_rng(32)
    for kscale, vscale, growth in ((1.0, 1.0, 9.0), (1e-20, 1e-20, 3.0), (1e3, 1e18, -9.0), (1e-3, 1e-2, 0.0)):
        n, new = 400, 24
        kvc, _, _, _ = paged(rng, [0], 1, 128, 32, 16, extra_pages=25, table_pages=25)
        kvc.page_table.copy_(torch.arange(25, dtype=torch.int32)[None])
        size = np.exp(np.linspace(0, growth, n)).astype(np.float32)[:, None, None]
        k, v = rows(rng, (n, 1), 128) * np.float32(kscale), rows(rng, (n, 1), 128) * np.float32(vscale) * size
        R.reskv_paged_append(kvc, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), torch.zeros(n, dtype=torch.int32, device="cuda"),
                             torch.arange(n, dtype=torch.int32, device="cuda"))
        ln = torch.tensor([n], dtype=torch.int32, device="cuda")
        kk, vv = (torch.empty((1, 1, n, 128), device="cuda") for _ in range(2))
        R.reskv_paged_gather(kvc, ln, kk, vv)
        q, q64 = as_type(rng.standard_normal((new, 4, 128)) / kscale, "bf16")
        o, lse = torch.empty((new, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((new, 4), device="cuda")
        R.reskv_paged_attn(kvc, q, ln, o, lse=lse)
        ref = po.attend(q64, kk[0].double().cpu().numpy(), vv[0].double().cpu().numpy(), 4, 128 ** -0.5)
        unit = vscale
        check(o.double() / unit, lse, [(ref[0] / unit, ref[1], ref[2], ref[3] / unit)], 128, "bf16")


def test_blocks_see_nothing_of_other_slots_and_later_tokens():
    """Garbage in unused slots, and NaN in tokens that only later queries see."""
    rng = np.random.default_rng(33)
    n, new, d, page = 150, 30, 128, 32
    kvc, values, pages, table = paged(rng, [n], 2, d, 32, page)
    q, q64 = as_type(rng.standard_normal((new, 8, d)), "bf16")
    ln = torch.tensor([n], dtype=torch.int32, device="cuda")
    o = torch.empty((new, 8, d), dtype=torch.bfloat16, device="cuda")
    R.reskv_paged_attn(kvc, q, ln, o)
    check(o, None, attend_all(values, q64, [0, new], 4, d ** -0.5, 0), d, "bf16")
    # position 140: values of group 1 are NaN in head 0, keys in head 1
    p = kvc.pages[int(table[0, 140 // page])].cpu().numpy()
    held = po.hold(rows(rng, (2,), d), 32)
    s16, m16 = held[1].copy(), held[2].copy()
    s16[0, 1] = m16[0, 1] = 0x7FC0
    s16[1, 2] = m16[1, 2] = 0x7FC0
    po.put_row(p, 0, 140 % page, d, 32, 1, held[0][0], s16[0], m16[0])
    po.put_row(p, 1, 140 % page, d, 32, 0, held[0][1], s16[1], m16[1])
    kvc.pages[int(table[0, 140 // page])] = torch.from_numpy(p).cuda()
    bad = torch.empty_like(o)
    R.reskv_paged_attn(kvc, q, ln, bad)
    first = new - (n - 140)                       # queries from here on see position 140
    assert torch.equal(bad[:first], o[:first])
    assert torch.isnan(bad[first:, :4, 32:64]).all() and torch.isfinite(bad[first:, :4, :32]).all() and torch.isfinite(bad[first:, :4, 64:]).all()
    assert torch.isnan(bad[first:, 4:]).all()
    kvc.check_status()


def test_blocks_report_faults():
    rng = np.random.default_rng(34)
    kvc, values, _, table = paged(rng, [200, 90], 1, 128, 32, 16)
    q, q64 = as_type(rng.standard_normal((40, 4, 128)), "bf16")
    o = torch.empty_like(q)
    ln = torch.tensor([200, 90], dtype=torch.int32, device="cuda")
    R.reskv_paged_attn(kvc, q, ln, o)
    kvc.check_status()
    check(o, None, attend_all(values, q64, [0, 20, 40], 4, 128 ** -0.5, 0), 128, "bf16")
    for page in (-1, len(kvc.pages)):
        kvc.page_table[0, 3] = page
        bad = torch.empty_like(q)
        R.reskv_paged_attn(kvc, q, ln, bad)
        with pytest.raises(R.ReskvError):
            kvc.check_status()
        # the missing page's positions are not seen, by this sequence alone
        keep = np.r_[0:48, 64:200]
        skip = [(values[0][0][:, keep], values[0][1][:, keep])]
        check(bad[:20], None, attend_all(skip, q64[:20], [0, 20], 4, 128 ** -0.5, 0), 128, "bf16")
        assert torch.equal(bad[20:], o[20:])


@pytest.mark.parametrize("ragged", [False, True])
def test_more_sequences_than_a_launch_takes(ragged):
    """2100 sequences: three launches of the few-row kernel, whose outputs equal those of the sequences apart."""
    B, kv, per, d = 2100, 1, 2, 64
    rng = np.random.default_rng(40)
    g = torch.Generator(device="cuda").manual_seed(1)
    lens = torch.from_numpy(rng.integers(0, 33, B).astype(np.int32)).cuda()
    pages = R.reskv_paged_pages(2 * B, kv, 16, d, 64)
    table = torch.randperm(2 * B, generator=g, device="cuda").to(torch.int32).view(B, 2)
    kvc = R.PagedKV(pages, table, 16, kv, d, 64)
    k, v = (torch.randn((B * 32, kv, d), generator=g, device="cuda") for _ in range(2))
    R.reskv_paged_append(kvc, k, v, torch.arange(B, dtype=torch.int32, device="cuda").repeat_interleave(32),
                         torch.arange(32, dtype=torch.int32, device="cuda").repeat(B))
    counts = rng.integers(0, 3, B) if ragged else np.ones(B, np.int64)
    begins = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    q = torch.randn((int(begins[-1]), kv * per, d), generator=g, device="cuda").bfloat16()
    o, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
    R.reskv_paged_attn(kvc, q, lens, o, q_begin=torch.from_numpy(begins).cuda() if ragged else None, lse=lse)
    kvc.check_status()
    for b in (0, 1, 1023, 1024, 1500, 2047, 2048, 2099):
        one = R.PagedKV(pages, table[b:b + 1].contiguous(), 16, kv, d, 64)
        s = slice(int(begins[b]), int(begins[b + 1]))
        if s.start == s.stop:
            continue
        want, ref = torch.empty_like(q[s]), torch.empty_like(lse[s])
        R.reskv_paged_attn(one, q[s], lens[b:b + 1].contiguous(), want, lse=ref)
        # the same tiles in the same order or in other pieces: a rounding of the output apart
        assert ((o[s].float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 1e-3).all()
        assert torch.allclose(lse[s], ref, atol=1e-3) or (lse[s] == ref).all()
    assert torch.isfinite(o).all()


@pytest.mark.parametrize("B,kv,new,length,window", [
    (12, 8, 16, 5000, 0),          # a part and a shorter one
    (2, 8, 260, 5000, 0),          # the same of 256 rows
    (31, 8, 16, 5000, 0),          # units of one CTA, and some in two parts
    (20, 8, 16, 2100, 0),          # units of one CTA, and some in four equal parts
    (31, 8, 16, 5000, 300),        # parts that see nothing
])
def test_blocks_in_parts_of_two_lengths(B, kv, new, length, window):
    """More units than the oracle takes: against the few-row kernel's fp32 output (query counts given), whose own
    share of the tolerance is added."""
    d, per, page = 128, 4, 64
    g = torch.Generator(device="cuda").manual_seed(B + new)
    n_pages = (length + page - 1) // page
    pages = R.reskv_paged_pages(B * n_pages, kv, page, d, 32)
    table = torch.randperm(B * n_pages, generator=g, device="cuda").to(torch.int32).view(B, n_pages)
    kvc = R.PagedKV(pages, table, page, kv, d, 32)
    for b in range(B):
        k, v = (torch.randn((length, kv, d), generator=g, device="cuda") for _ in range(2))
        R.reskv_paged_append(kvc, k, v, torch.full((length,), b, dtype=torch.int32, device="cuda"),
                             torch.arange(length, dtype=torch.int32, device="cuda"))
    lens = torch.tensor([max(new, length - 97 * b) for b in range(B)], dtype=torch.int32, device="cuda")
    q = torch.randn((B * new, kv * per, d), generator=g, device="cuda").bfloat16()
    o, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
    R.reskv_paged_attn(kvc, q, lens, o, lse=lse, window=window)
    ref, ref_lse = torch.empty(q.shape, device="cuda"), torch.empty_like(lse)
    begins = (torch.arange(B + 1, device="cuda") * new).to(torch.int32)
    R.reskv_paged_attn(kvc, q, lens, ref, q_begin=begins, lse=ref_lse, window=window)
    kvc.check_status()
    kk, vv = (torch.empty((B, kv, length, d), device="cuda") for _ in range(2))
    R.reskv_paged_gather(kvc, lens, kk, vv)
    x = d ** -0.5 * (q.float().view(B, new, kv, per, d).abs().amax((1, 3, 4)) * kk.abs().sum(-1).amax(-1)).max().item()
    tol = 2 * (2 * d * 2.0 ** -23 * x + 2.0 ** -11 + 2.0 ** -16) * vv.abs().max().item() + HALF_ULP["bf16"] * ref.abs() * 1.01 + 1e-7
    assert ((o.float() - ref).abs() <= tol).all()
    assert ((lse - ref_lse).abs() <= 2 * (d * 2.0 ** -23 * x + 2.0 ** -12 + 2.0 ** -22 * ref_lse.abs())).all()
    again = torch.empty_like(o)
    R.reskv_paged_attn(kvc, q, lens, again, window=window)
    assert torch.equal(o, again)


def test_offsets_beyond_32_bits():
    """A cache of 5 GB whose last pages are used, against the same tokens in one of a few pages."""
    d, kv, per, page, n = 128, 8, 4, 64, 200
    g = torch.Generator(device="cuda").manual_seed(2)
    used = (n + page - 1) // page
    page_bytes = R.reskv_paged_pages(1, kv, page, d, 32).numel()
    n_pages = (5 << 30) // page_bytes
    far = torch.empty((n_pages, page_bytes), dtype=torch.uint8, device="cuda")
    table = (n_pages - 1 - torch.arange(used, device="cuda", dtype=torch.int32))[None].contiguous()
    big = R.PagedKV(far, table, page, kv, d, 32)
    small = R.PagedKV(R.reskv_paged_pages(used, kv, page, d, 32), torch.arange(used, device="cuda", dtype=torch.int32)[None],
                      page, kv, d, 32)
    k, v = (torch.randn((n, kv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    seqs, pos = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    outs = []
    for kvc in (big, small):
        R.reskv_paged_append(kvc, k, v, seqs, pos)
        kk, vv = (torch.empty((1, kv, n, d), device="cuda") for _ in range(2))
        R.reskv_paged_gather(kvc, lens, kk, vv)
        outs.append([kk, vv])
        for new in (1, 20):                             # the kernel of few rows, that of many
            q = torch.randn((new, kv * per, d), generator=torch.Generator(device="cuda").manual_seed(new), device="cuda").bfloat16()
            outs[-1].append(torch.empty_like(q))
            R.reskv_paged_attn(kvc, q, lens, outs[-1][-1])
        kvc.check_status()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
