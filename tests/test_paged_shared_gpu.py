"""Attention with a shared prefix against fp64: tolerance as for reskv_paged_attn (logits summed in fp32,
weights of 11 bits at least, half a unit of the output's type), the weights of the joined
parts within 2^-18 beside."""
import numpy as np
import pytest
import torch

from oracle import cross_oracle as co
from paged_cases import DT, HALF_ULP, as_type, paged
from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu


def check(o, lse, refs, d, dtype):
    ro, rl, xm, vm = (np.concatenate([r[i] for r in refs]) for i in range(4))
    got = o.double().cpu().numpy()
    share = 2 * d * 2.0 ** -23 * xm + 2.0 ** -11 + 2.0 ** -16 + (2.0 ** -11 if dtype != "f32" else 0)      # weights and held values
    tol = (share * vm)[..., None] + HALF_ULP[dtype] * np.abs(ro) * 1.01 + 1e-7
    assert np.isfinite(got).all()
    assert (np.abs(got - ro) <= tol).all(), (np.abs(got - ro) - tol).max()
    gl = lse.double().cpu().numpy()
    assert ((gl == -np.inf) == (rl == -np.inf)).all()
    seen = rl != -np.inf
    bound = d * 2.0 ** -23 * xm + 2.0 ** -12 + 2.0 ** -22 * np.abs(np.where(seen, rl, 0))
    assert (np.abs(gl[seen] - rl[seen]) <= bound[seen]).all()


def case(seed, prefix_lens, lens, members, new, kv=2, per=4, d=128, group=32, page=32, dtype="bf16", out=None, counts=None,
         scale=None, uniform=False):
    """members: sequences of every group; counts: query tokens of every sequence (None: new each)."""
    rng = np.random.default_rng(seed)
    prefix, pv, _, _ = paged(rng, prefix_lens, kv, d, group, page)
    own, ov, _, _ = paged(rng, lens, kv, d, group, page)
    B, H = len(lens), kv * per
    n = counts if counts is not None else [new] * B
    begins = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    at = np.concatenate([[0], np.cumsum(members)]).astype(np.int32)
    q, q64 = as_type(rng.standard_normal((begins[-1], H, d)), dtype)
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    a = dict(seq_begin=None if uniform else ints(at), q_begin=None if counts is None else ints(begins), scale=scale)

    def run():
        o = torch.full((begins[-1], H, d), float("nan"), dtype=DT[out or dtype], device="cuda")
        lse = torch.full((begins[-1], H), float("nan"), device="cuda")
        R.reskv_paged_attn_shared(own, prefix, q, ints(lens), ints(prefix_lens), o, lse=lse, **a)
        own.check_status()
        prefix.check_status()
        return o, lse

    o, lse = run()
    refs = []
    for b in range(B):
        g = int(np.searchsorted(at, b, "right")) - 1
        pk, pvv = pv[g] if g < len(prefix_lens) else (np.zeros((kv, 0, d)),) * 2
        k, v = np.concatenate([pk, ov[b][0]], 1), np.concatenate([pvv, ov[b][1]], 1)
        t = np.arange(k.shape[1])
        upto = pk.shape[1] + lens[b] - n[b] + np.arange(n[b])
        see = (t <= upto[:, None]) | (t < pk.shape[1])
        see &= (t < pk.shape[1]) | (t <= upto[:, None])
        refs.append(co.attend(q64[begins[b]:begins[b + 1]], k, v, d ** -0.5 if scale is None else scale, see))
    check(o, lse, refs, d, out or dtype)
    o2, lse2 = run()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("d,group", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("batch", [3, 20, 33])
def test_single_tokens(d, group, dtype, batch):
    lens = [1 + (37 * i) % 90 for i in range(batch)]
    case(1, [150], lens, [batch], 1, d=d, group=group, dtype=dtype)


@pytest.mark.parametrize("prefix", [0, 1, 15, 16, 17, 64, 65, 700])
@pytest.mark.parametrize("batch,per", [(2, 2), (40, 2), (40, 4)])
def test_prefix_lengths(prefix, batch, per):
    case(prefix, [prefix], [5 + i for i in range(batch)], [batch], 1, per=per)


@pytest.mark.parametrize("per", [1, 3, 7, 16])
@pytest.mark.parametrize("batch", [4, 33])
def test_head_groups(per, batch):
    case(per, [90], [3 + 2 * i for i in range(batch)], [batch], 1, kv=3, per=per, d=64, group=32)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_several_groups(dtype):
    case(2, [100, 0, 333, 17], [9, 30, 1, 64, 65, 2, 70, 40, 8, 3], [1, 4, 3, 2], 1, dtype=dtype)
    case(3, [100, 0, 333, 17], [9 + i for i in range(70)], [20, 0, 30, 20], 1, dtype=dtype)
    case(3, [100, 0, 333, 17], [9 + i for i in range(70)], [20, 0, 30, 20], 1, per=8, dtype=dtype)
    case(4, [64, 200], [20] * 40, [20, 20], 1, uniform=True, dtype=dtype)
    case(4, [64, 200], [20] * 40, [20, 20], 1, per=7, uniform=True, dtype=dtype)
    case(5, [50], [9, 30, 12], [2], 1, dtype=dtype)                    # the last sequence is in no group


@pytest.mark.parametrize("new", [2, 5, 16])
@pytest.mark.parametrize("batch", [1, 9])
def test_several_tokens(new, batch):
    case(new, [140], [new + 7 * i for i in range(batch)], [batch], new)
    case(new + 1, [140, 30], [new + 7 * i for i in range(batch + 1)], [batch, 1], new, dtype="f16", d=64, group=64)
    case(new + 2, [140], [new + 7 * i for i in range(batch)], [batch], new, per=64)


def test_ragged_queries_and_tokens_before_the_own_ones():
    case(6, [120, 60], [20, 9, 64, 3, 30], [3, 2], None, counts=[2, 0, 7, 3, 1])
    case(6, [120, 60], [20, 9, 64, 3, 30], [3, 2], None, counts=[2, 0, 7, 3, 1], per=24)
    case(7, [120, 60], [1, 0, 2], [2, 1], 3, per=32)
    case(7, [120, 60], [1, 0, 2], [2, 1], 3)                            # some stand before their own tokens
    case(8, [0, 60], [1, 0, 2], [2, 1], 3)                              # and see nothing
    case(9, [120], [40] * 4, [4], None, counts=[30, 1, 60, 0])


def test_chunks_of_own_tokens():
    """So many new tokens that both passes go by blocks of rows."""
    case(10, [300], [80, 64], [2], 64)
    case(11, [300, 70], [64, 64, 64, 64], [1, 3], 40, dtype="f16", uniform=False)


def test_outputs_in_fp32_and_scale():
    case(12, [200], [50, 60, 1], [3], 1, out="f32")
    case(13, [200], [50 + i for i in range(30)], [30], 1, out="f32", dtype="f16", d=64, scale=0.05)


def test_agrees_with_one_long_sequence():
    """A prefix and own tokens in one sequence's pages, through reskv_paged_attn."""
    rng = np.random.default_rng(14)
    kv, per, d, page = 2, 4, 128, 16
    whole, _, _, table = paged(rng, [96 + 21, 96 + 40], kv, d, 32, page)
    # sequence 0's first six pages are the prefix of both
    t = torch.from_numpy(table).cuda()
    whole.page_table[1, :6] = t[0, :6]
    lens = torch.tensor([21, 40], dtype=torch.int32, device="cuda")
    prefix = R.PagedKV(whole.pages, t[:1, :6].contiguous(), page, kv, d, 32)
    own = R.PagedKV(whole.pages, t[:, 6:].contiguous(), page, kv, d, 32)
    q, _ = as_type(rng.standard_normal((2, kv * per, d)), "f16")
    a, b = (torch.empty(q.shape, device="cuda") for _ in range(2))
    R.reskv_paged_attn(whole, q, lens + 96, a)
    R.reskv_paged_attn_shared(own, prefix, q, lens, torch.tensor([96], dtype=torch.int32, device="cuda"), b)
    for kvc in (whole, own, prefix):
        kvc.check_status()
    assert float((a - b).abs().max()) <= 2.0 ** -16 * 40              # two fp32 results, values within 40


@pytest.mark.parametrize("batch", [3, 20, 33])
def test_long_prefixes(batch):
    """Many tiles a CTA, for one block of rows and for two."""
    case(17, [3000], [4 + i for i in range(batch)], [batch], 1, kv=1, per=4, group=64)
    case(18, [2500, 40], [4 + i for i in range(2 * batch)], [batch, batch], 1, kv=1, per=16, d=64, group=32, dtype="f16")


@pytest.mark.parametrize("batch,scale", [(40, 1e-20), (40, 1e9), (3, 1e9), (64, 1e-20), (64, 1e9)])
def test_values_and_keys_of_any_size(batch, scale):
    """Tokens far larger and far smaller than their neighbours, in keys that queries avoid and in values."""
    rng = np.random.default_rng(19)
    kv, d, n = 1, 128, 200
    prefix, _, _, _ = paged(rng, [0], kv, d, 32, 16, extra_pages=13, table_pages=13)
    prefix.page_table.copy_(torch.arange(13, dtype=torch.int32)[None])
    own, _, _, _ = paged(rng, [0] * batch, kv, d, 32, 16, extra_pages=batch, table_pages=1)
    own.page_table.copy_(torch.arange(batch, dtype=torch.int32)[:, None])
    k, v = rng.standard_normal((2, n, kv, d)).astype(np.float32) * np.float32(scale)
    k[..., 0], v[7::16] = 0, v[7::16] * 1e8                               # channel 0 alone tells the large keys
    k[7::16] = 0
    k[7::16, :, 0] = -60 * scale
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    kt, vt = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda()
    R.reskv_paged_append(prefix, kt, vt, ints(np.zeros(n)), ints(np.arange(n)))
    R.reskv_paged_append(own, kt[:batch].contiguous(), vt[:batch].contiguous(), ints(np.arange(batch)), ints(np.zeros(batch)))
    held = [torch.empty((1, kv, n, d), device="cuda") for _ in range(2)]
    R.reskv_paged_gather(prefix, ints([n]), *held)
    mine = [torch.empty((batch, kv, 1, d), device="cuda") for _ in range(2)]
    R.reskv_paged_gather(own, ints(np.ones(batch)), *mine)
    q = rng.standard_normal((batch, 2, d)) / scale
    q[..., 0] = 20 / scale                                                # the large tokens' weights vanish
    q, q64 = as_type(q, "bf16")
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    R.reskv_paged_attn_shared(own, prefix, q, ints(np.ones(batch)), ints([n]), o, lse=lse)
    for kvc in (own, prefix):
        kvc.check_status()
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    for b in range(batch):
        kk, vv = (np.concatenate([f64(h[0]), f64(m[b])], 1) for h, m in zip(held, mine))
        ro, rl, xm, _ = co.attend(q64[b:b + 1], kk, vv, d ** -0.5)
        # in units of the values that count: weights of the large ones are below 2^-100
        small = np.abs(vv[:, np.abs(vv).max((0, 2)) < 100 * scale]).max()
        share = 2 * d * 2.0 ** -23 * xm + 2.0 ** -10 + 2.0 ** -16
        tol = (share * small)[..., None] + HALF_ULP["bf16"] * np.abs(ro) * 1.01 + 2.0 ** -120
        worst = (np.abs(f64(o)[b:b + 1] - ro) - tol).max() / small
        assert worst <= 0
        assert (np.abs(f64(lse)[b:b + 1] - rl) <= d * 2.0 ** -23 * xm + 2.0 ** -12 + 2.0 ** -22 * np.abs(rl)).all()


@pytest.mark.parametrize("batch", [3, 24, 40])
def test_nan_held_in_a_prefix_reaches_its_group_alone(batch):
    rng = np.random.default_rng(20)
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    prefix, _, pages, table = paged(rng, [70, 50], 1, 128, 32, 16)
    own, _, _, _ = paged(rng, [9] * 2 * batch, 1, 128, 32, 16)
    bad = torch.zeros((1, 1, 128), device="cuda")
    bad[..., 40] = float("nan")
    good = torch.zeros_like(bad)
    R.reskv_paged_append(prefix, good, bad, ints([1]), ints([33]))
    q, _ = as_type(rng.standard_normal((2 * batch, 4, 128)), "bf16")
    o = torch.empty_like(q)
    R.reskv_paged_attn_shared(own, prefix, q, ints([9] * 2 * batch), ints([70, 50]), o)
    nan = torch.isnan(o)
    assert not nan[:batch].any()
    assert nan[batch:, :, 32:64].all() and not nan[batch:, :, :32].any() and not nan[batch:, :, 64:].any()
    # behind the prefix's end it is nobody's
    R.reskv_paged_attn_shared(own, prefix, q, ints([9] * 2 * batch), ints([70, 33]), o)
    assert not torch.isnan(o).any()


@pytest.mark.parametrize("batch", [3, 24, 40])
def test_pages_past_32_bits(batch):
    """The same prefix in the first and in the last pages of more than 4 GB."""
    rng = np.random.default_rng(21)
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    near, _, pages, table = paged(rng, [130], 2, 128, 32, 64)
    own, _, _, _ = paged(rng, [5] * batch, 2, 128, 32, 64)
    n = (1 << 32) // pages[0].size + 10
    big = torch.zeros((n, *pages.shape[1:]), dtype=torch.uint8, device="cuda")
    last = ints([[n - 1, n - 3, n - 2]])
    big[last[0].long()] = near.pages[near.page_table[0, :3].long()]
    far = R.PagedKV(big, last, 64, 2, 128, 32)
    q, _ = as_type(rng.standard_normal((batch, 8, 128)), "f16")
    a, b = torch.empty_like(q), torch.empty_like(q)
    R.reskv_paged_attn_shared(own, near, q, ints([5] * batch), ints([130]), a)
    R.reskv_paged_attn_shared(own, far, q, ints([5] * batch), ints([130]), b)
    far.check_status()
    assert torch.equal(a, b)


@pytest.mark.parametrize("batch", [3, 24, 40])
def test_any_rows_of_queries_and_outputs(batch):
    """Strided and unaligned queries and outputs, the same bits."""
    rng = np.random.default_rng(22)
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    prefix, _, _, _ = paged(rng, [100], 2, 64, 32, 16)
    own, _, _, _ = paged(rng, [5] * batch, 2, 64, 32, 16)
    q, _ = as_type(rng.standard_normal((batch, 8, 64)), "bf16")
    want = torch.empty_like(q)
    R.reskv_paged_attn_shared(own, prefix, q, ints([5] * batch), ints([100]), want)
    for pad in (1, 8):
        wide = torch.zeros((batch, 8, 64 + pad), dtype=q.dtype, device="cuda")
        wide[..., :64] = q
        out = torch.zeros_like(wide)
        R.reskv_paged_attn_shared(own, prefix, wide[..., :64], ints([5] * batch), ints([100]), out[..., :64])
        assert torch.equal(out[..., :64], want) and (out[..., 64:] == 0).all()


def test_faults_are_reported_and_bounded():
    rng = np.random.default_rng(15)
    prefix, _, _, _ = paged(rng, [60, 60], 2, 128, 32, 32)
    own, _, _, _ = paged(rng, [20] * 30, 2, 128, 32, 32)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, _ = as_type(rng.standard_normal((30, 8, 128)), "bf16")
    o = torch.empty_like(q)
    for seqs, lens in (([0, 15, 30], [60, 1000]), ([0, 15, 30], [-1, 60]), ([0, 15, 300], [60, 60]), ([-4, 15, 30], [60, 60]),
                       ([0, 30, 0], [60, 60]), ([30, 0, 30], [60, 60])):
        R.reskv_paged_attn_shared(own, prefix, q, ints([20] * 30), ints(lens), o, seq_begin=ints(seqs))
        with pytest.raises(R.ReskvError, match="index"):
            prefix.check_status()
        own.check_status()


@pytest.mark.parametrize("batch", [3, 24, 40])
def test_captured_call_replayed(batch):
    rng = np.random.default_rng(16)
    prefix, _, _, _ = paged(rng, [200], 2, 128, 32, 32)
    own, _, _, _ = paged(rng, [50] * batch, 2, 128, 32, 32)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, _ = as_type(rng.standard_normal((batch, 8, 128)), "bf16")
    o, lens, plens = torch.empty_like(q), ints([50] * batch), ints([200])
    ws = torch.zeros(R.reskv_paged_attn_shared_workspace(own, prefix, batch, 8), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        R.reskv_paged_attn_shared(own, prefix, q, lens, plens, o, workspace=ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        R.reskv_paged_attn_shared(own, prefix, q, lens, plens, o, workspace=ws)
    q.mul_(0.5)
    lens.copy_(ints([7 + i for i in range(batch)]))
    plens.fill_(99)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    got = o.clone()
    R.reskv_paged_attn_shared(own, prefix, q, lens, plens, o)
    assert torch.equal(got, o)


@pytest.mark.parametrize("batch", [3, 40])
def test_calls_behind_writes_of_all_that_they_read(batch):
    """Tables, lengths, groups, queries and rows that kernels just before write, call after call without a pause."""
    rng = np.random.default_rng(23)
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    two, _, _, _ = paged(rng, [1504, 1504], 2, 128, 32, 32)
    own, _, _, _ = paged(rng, [30] * batch, 2, 128, 32, 32)
    prefix = R.PagedKV(two.pages, two.page_table.clone(), 32, 2, 128, 32)
    tables = torch.stack([two.page_table, two.page_table.flip(0), two.page_table.roll(1, 1)])
    steps = 24
    qs, _ = as_type(rng.standard_normal((steps, batch, 8, 128)), "bf16")
    rows, _ = as_type(rng.standard_normal((steps, 2, 2, 2, 128)), "bf16")
    lens, plens = ints(rng.integers(1, 31, (steps, batch))), ints(rng.integers(1, 1505, (steps, 2)))
    at = ints(np.stack([np.zeros(steps), rng.integers(0, batch + 1, steps), np.full(steps, batch)], 1))
    q, n, pn, begin = torch.empty_like(qs[0]), torch.empty_like(lens[0]), torch.empty_like(plens[0]), torch.empty_like(at[0])
    start, last, which = two.pages.clone(), torch.empty_like(plens[0]), ints([0, 1])
    torch.cuda.synchronize()

    def all_steps(pause):
        two.pages.copy_(start)
        outs = torch.full_like(qs, float("nan"))
        for i in range(steps):
            for to, source in ((q, qs[i]), (n, lens[i]), (pn, plens[i]), (begin, at[i]), (prefix.page_table, tables[i % 3])):
                torch.add(source, 0, out=to)
            torch.sub(pn, 1, out=last)
            R.reskv_paged_append(prefix, rows[i, 0], rows[i, 1], which, last)
            pause()
            R.reskv_paged_attn_shared(own, prefix, q, n, pn, outs[i], seq_begin=begin)
            pause()
        own.check_status()
        prefix.check_status()
        return outs

    want = all_steps(torch.cuda.synchronize)
    assert torch.isfinite(want.float()).all()
    for _ in range(3):
        assert torch.equal(all_steps(lambda: None), want)
