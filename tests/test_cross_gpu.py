"""Cross attention and its gradient against fp64.

Tolerance, from the number formats.  A logit is a sum of d products in fp32, off by
at most d 2^-23 X with X = scale sum |q k|; a weight is then off by a factor of at most
1 + 2 d 2^-23 X, and by half a step of the type where it is rounded to it; the sums
over states add 2^-16.  An output, a mean of values, is off by at most that share of
the largest |v|, then half a step of its type.  The gradient's bounds are in
oracle.cross_oracle.gradient.
"""
import numpy as np
import pytest
import torch

from oracle import cross_oracle as co
from paged_cases import DT, HALF_ULP, as_type
from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu

LEAST = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25}        # half a smallest step


def check(o, lse, refs, d, dtype):
    ro, rl, xm, vm = (np.concatenate([r[i] for r in refs]) for i in range(4))
    got = o.double().cpu().numpy()
    share = 2 * d * 2.0 ** -23 * xm + HALF_ULP[dtype] + 2.0 ** -16
    tol = (share * vm)[..., None] + HALF_ULP[dtype] * np.abs(ro) * 1.01 + LEAST[dtype] + 1e-7 * vm[..., None]
    assert np.isfinite(got).all()
    worst = (np.abs(got - ro) - tol).max()
    assert worst <= 0
    gl = lse.double().cpu().numpy()
    assert ((gl == -np.inf) == (rl == -np.inf)).all()
    seen = rl != -np.inf
    if seen.any():
        bound = d * 2.0 ** -23 * xm + 2.0 ** -16 + 2.0 ** -22 * np.abs(np.where(seen, rl, 0))
        worst = (np.abs(gl[seen] - rl[seen]) - bound[seen]).max()
        assert worst <= 0


def spans(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


class Case:
    """counts query tokens and lens states a sequence; form: equal, padded (to `pad` rows) or packed; gap: rows
    and tokens before the first sequence and after the last (packed).  Rows that nobody sees are NaN."""

    def __init__(self, seed, counts, lens, kv, per, d, dtype, form="packed", pad=None, gap=0, spread=1.0, scale=None,
                 fused=False, offset=0):
        rng = np.random.default_rng(seed)
        self.counts, self.lens, self.kv, self.per, self.d, self.dtype = counts, lens, kv, per, d, dtype
        self.scale = scale
        B, H = len(counts), kv * per
        self.args = dict(batch=B)
        if form == "packed":
            qb, kb = spans(counts) + gap, spans(lens) + gap
            T, rows = int(qb[-1]) + gap, int(kb[-1]) + gap
            self.args.update(q_begin=torch.from_numpy(qb).cuda(), kv_begin=torch.from_numpy(kb).cuda())
        else:
            pad = max(max(lens), 1) if pad is None else pad
            qb, kb = spans(counts), (np.arange(B + 1) * pad).astype(np.int32)
            T, rows = int(qb[-1]), B * pad
            assert len(set(counts)) == 1
            if form == "padded":
                self.args.update(kv_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
            else:
                assert set(lens) == {pad}
        self.qb, self.kb, self.T, self.rows = qb, kb, T, rows
        k, v = rng.standard_normal((2, rows, kv, d)) * spread
        q = rng.standard_normal((T, H, d))
        self.seen_rows, self.seen_tokens = np.zeros(rows, bool), np.zeros(T, bool)
        for b in range(B):
            self.seen_rows[kb[b]:kb[b] + lens[b]] = True
            self.seen_tokens[qb[b]:qb[b] + counts[b]] = True
        k[~self.seen_rows], v[~self.seen_rows] = np.nan, np.nan
        q[~self.seen_tokens] = np.nan
        self.q, self.q64 = self.place(q, offset)
        if fused:                                  # keys and values out of one projection
            both, both64 = self.place(np.concatenate([k, v], 1), offset)
            self.k, self.v, self.k64, self.v64 = both[:, :kv], both[:, kv:], both64[:, :kv], both64[:, kv:]
        else:
            (self.k, self.k64), (self.v, self.v64) = self.place(k, offset), self.place(v, offset)
        self.g, self.g64 = self.place(np.where(self.seen_tokens[:, None, None], rng.standard_normal((T, H, d)), np.nan), offset)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def place(self, x, offset):
        """The tensor, `offset` elements off its allocation's boundary."""
        t, x64 = as_type(x, self.dtype)
        if offset:
            flat = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
            flat[offset:] = t.flatten()
            t = flat[offset:].view(t.shape)
        return t, x64

    def sequences(self):
        for b, n in enumerate(self.counts):
            q0, k0 = self.qb[b], self.kb[b]
            yield slice(q0, q0 + n), slice(k0, k0 + self.lens[b]), slice(k0, self.kb[b + 1])

    def forward(self, fill=float("nan")):
        o = torch.full((self.T, self.kv * self.per, self.d), fill, dtype=DT[self.dtype], device="cuda")
        lse = torch.full(o.shape[:2], fill, device="cuda")
        R.reskv_cross_attn(self.q, self.k, self.v, o, scale=self.scale, lse=lse, status=self.status, **self.args)
        return o, lse

    def backward(self, o, lse, fill=7.0, like=None):
        dq = torch.full_like(self.q, fill)
        dk, dv = (torch.full((self.rows, self.kv, self.d), fill, dtype=DT[self.dtype], device="cuda") for _ in range(2))
        if like == "fused":
            both = torch.full((self.rows, 2 * self.kv, self.d), fill, dtype=DT[self.dtype], device="cuda")
            dk, dv = both[:, :self.kv], both[:, self.kv:]
        R.reskv_cross_attn_backward(self.q, self.k, self.v, o, lse, self.g, dq, dk, dv, scale=self.scale,
                                    status=self.status, **self.args)
        return dq, dk, dv

    def check(self, train=True):
        scale = self.d ** -0.5 if self.scale is None else self.scale
        o, lse = self.forward()
        refs = [co.attend(self.q64[t], self.k64[r].transpose(1, 0, 2), self.v64[r].transpose(1, 0, 2), scale)
                for t, r, _ in self.sequences()]
        check(o[torch.from_numpy(self.seen_tokens)], lse[torch.from_numpy(self.seen_tokens)], refs, self.d, self.dtype)
        assert torch.isnan(o[torch.from_numpy(~self.seen_tokens)]).all()          # tokens of no sequence are left
        again, lse2 = self.forward()
        assert torch.equal(o.view(torch.int16), again.view(torch.int16)) and torch.equal(lse.view(torch.int32), lse2.view(torch.int32))
        if not train:
            assert int(self.status) == 0
            return
        grads = self.backward(o, lse)
        dq, dk, dv = (x.double().cpu().numpy() for x in grads)
        owned = np.zeros(self.rows, bool)
        for t, r, whole in self.sequences():
            owned[whole] = True
            ref, tol = co.gradient(self.q64[t], self.k64[r].transpose(1, 0, 2), self.v64[r].transpose(1, 0, 2), self.g64[t], scale,
                                   HALF_ULP[self.dtype], LEAST[self.dtype])
            for name, got, want, off in (("dq", dq[t], ref[0], tol[0]), ("dk", dk[r].transpose(1, 0, 2), ref[1], tol[1]),
                                         ("dv", dv[r].transpose(1, 0, 2), ref[2], tol[2])):
                assert np.isfinite(got).all(), name
                worst = (np.abs(got - want) - off * 1.01).max(initial=0.0)
                assert worst <= 0, name
            # rows of the sequence that nobody sees
            assert (dk[r.stop:whole.stop] == 0).all() and (dv[r.stop:whole.stop] == 0).all()
        assert (dk[~owned] == 7).all() and (dv[~owned] == 7).all() and (dq[~self.seen_tokens] == 7).all()
        for x, y in zip(grads, self.backward(o, lse)):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))
        assert int(self.status) == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("counts,lens", [([1], [1]), ([1, 1, 1, 1], [17, 0, 64, 200]), ([3, 0, 5], [129, 40, 128]),
                                         ([40, 33], [1, 130]), ([130, 1, 257], [257, 300, 127])])
def test_packed(d, dtype, counts, lens):
    Case(1, counts, lens, 2, 2, d, dtype).check()


@pytest.mark.parametrize("per", [1, 3, 4, 7, 8, 16, 64])
@pytest.mark.parametrize("n", [1, 5, 40])
def test_head_groups(per, n):
    Case(per, [n, n], [70, 133], 2, per, 64 if per > 4 else 128, "bf16").check()


@pytest.mark.parametrize("n", [1, 2, 9, 64, 150])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f16")])
def test_padded_batches(n, d, dtype):
    Case(n, [n] * 4, [100, 0, 161, 7], 2, 4, d, dtype, form="padded", pad=161).check()


def test_equal_sequences():
    Case(2, [20] * 3, [90] * 3, 3, 2, 128, "bf16", form="equal").check()
    Case(3, [1] * 3, [256] * 3, 3, 1, 64, "f16", form="equal").check()


@pytest.mark.parametrize("n", [1, 33])
def test_rows_around_the_sequences_are_left(n):
    Case(4, [n, n + 1], [60, 131], 2, 2, 128, "bf16", gap=5).check()
    Case(4, [n, n + 1], [60, 131], 2, 2, 64, "f16", gap=3).check()


@pytest.mark.parametrize("n", [1, 30])
def test_keys_and_values_of_one_projection(n):
    c = Case(5, [n, n], [100, 150], 2, 4, 128, "bf16", fused=True)
    c.check()
    o, lse = c.forward()
    for x, y in zip(c.backward(o, lse), c.backward(o, lse, like="fused")):
        assert torch.equal(x, y)


@pytest.mark.parametrize("n", [1, 30])
@pytest.mark.parametrize("offset", [1, 4])
def test_any_alignment(n, offset):
    Case(6, [n, n], [65, 150], 2, 2, 128, "bf16", offset=offset).check()
    Case(6, [n, n], [65, 150], 1, 4, 64, "f16", offset=offset, fused=True).check()


@pytest.mark.parametrize("n", [1, 40, 150])
def test_peaked_and_flat_queries(n):
    Case(7, [n], [300], 1, 2, 128, "bf16", scale=1.0).check()
    Case(8, [n], [300], 1, 2, 64, "f16", scale=3.0).check()
    Case(9, [n], [300], 1, 2, 64, "bf16", scale=1e-4).check()
    Case(10, [n], [300], 1, 2, 64, "bf16", scale=-0.3).check()


def test_negative_scale_of_either_type():
    Case(18, [40], [300], 1, 2, 64, "f16", scale=-0.4).check()
    Case(19, [2], [300], 1, 2, 128, "f16", scale=-0.4).check()


@pytest.mark.parametrize("n", [1, 50])
def test_heads_before_tokens(n):
    """Rows as [head, token, dim] and with gaps: the same bits as from packed rows."""
    c = Case(20, [n, n], [200, 131], 2, 4, 128, "bf16", form="padded", pad=200)
    o, lse = c.forward()
    grads = c.backward(o, lse)
    turned = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    wide = lambda t: torch.cat([t, t, t], 2)[:, :, :t.shape[2]]  # noqa: E731
    for lay in (turned, wide):
        q, k, v, g = (lay(t) for t in (c.q, c.k, c.v, c.g))
        o2, lse2 = lay(torch.zeros_like(o)), torch.zeros_like(lse)
        assert o2.stride() != o.stride() or n == 1
        R.reskv_cross_attn(q, k, v, o2, lse=lse2, **c.args)
        assert torch.equal(o2, o) and torch.equal(lse2, lse)
        out = [lay(torch.zeros_like(t)) for t in grads]
        R.reskv_cross_attn_backward(q, k, v, o2, lse2, g, *out, **c.args)
        for a, b in zip(out, grads):
            assert torch.equal(a, b)


@pytest.mark.parametrize("n", [2, 60])
def test_broadcast_heads(n):
    """One head of keys and values for all (a head stride of 0), the general path, against the same rows copied."""
    c = Case(21, [n], [90], 1, 1, 64, "bf16")
    q = torch.randn((n, 4, 64), device="cuda").bfloat16()
    one, four = c.k.expand(-1, 4, -1), c.k.repeat(1, 4, 1)
    a, b = torch.empty_like(q), torch.empty_like(q)
    R.reskv_cross_attn(q, one, one, a)
    R.reskv_cross_attn(q, four, four, b)
    assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -7 * 5            # two roundings each of values within 5


def test_no_states_and_no_tokens():
    q, none = torch.randn((3, 4, 64), device="cuda").half(), torch.empty((0, 2, 64), dtype=torch.float16, device="cuda")
    o, lse, dq = torch.full_like(q, 7), torch.zeros((3, 4), device="cuda"), torch.full_like(q, 7)
    R.reskv_cross_attn(q, none, none, o, lse=lse)
    assert (o == 0).all() and (lse == -np.inf).all()
    R.reskv_cross_attn_backward(q, none, none, o, lse, q, dq, none, none)
    assert (dq == 0).all()
    k = torch.randn((5, 2, 64), device="cuda").half()
    empty, dk, dv = q[:0], torch.full_like(k, 7), torch.full_like(k, 7)
    R.reskv_cross_attn(empty, k, k, empty, lse=lse[:0])
    R.reskv_cross_attn_backward(empty, k, k, empty, lse[:0], empty, empty, dk, dv)
    assert (dk == 0).all() and (dv == 0).all()


@pytest.mark.parametrize("n", [1, 40])
def test_offsets_past_32_bits(n):
    """Rows 2^20 elements apart: 3000 of them reach past 2^31 elements and 2^32 bytes."""
    c = Case(22, [n], [3000], 1, 2, 128, "bf16", form="equal", pad=3000)
    o, lse = c.forward()
    grads = c.backward(o, lse)
    far = lambda: torch.empty(3000 << 20, dtype=torch.bfloat16, device="cuda").as_strided((3000, 1, 128), (1 << 20, 128, 1))  # noqa: E731
    k, v, dk, dv = far(), far(), far(), far()
    k.copy_(c.k)
    v.copy_(c.v)
    o2, lse2, dq = torch.empty_like(o), torch.empty_like(lse), torch.empty_like(o)
    R.reskv_cross_attn(c.q, k, v, o2, lse=lse2)
    R.reskv_cross_attn_backward(c.q, k, v, o2, lse2, c.g, dq, dk, dv)
    assert torch.equal(o2, o) and torch.equal(dq, grads[0]) and torch.equal(dk, grads[1]) and torch.equal(dv, grads[2])


def test_two_streams_at_once():
    cases = [Case(23 + i, [n], [700], 2, 2, 128, "bf16") for i, n in enumerate((1, 30, 300))]
    want = [(c.forward(), c) for c in cases]
    want = [(f, c.backward(*f)) for f, c in want]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = []
    for _ in range(4):
        got = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                f = c.forward()
                got.append((f, c.backward(*f)))
    torch.cuda.synchronize()
    for (f, g), (f2, g2) in zip(want, got):
        for a, b in zip((*f, *g), (*f2, *g2)):
            assert torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float()))


def test_longer_states():
    Case(11, [1, 2], [3000, 1111], 2, 4, 128, "bf16").check()
    Case(12, [70], [1500], 2, 1, 64, "f16").check()


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f16")])
@pytest.mark.parametrize("counts,lens", [([3], [3000]), ([20, 3], [2100, 700]), ([700], [60]), ([300, 1], [50, 400]), ([300], [1100])])
def test_few_blocks_shared_by_clusters(d, dtype, counts, lens):
    Case(17, counts, lens, 1, 4, d, dtype).check()


def test_gradient_against_differences():
    """<d_o, o(q + h u) - o(q - h u)> / 2h along random directions, o from the oracle."""
    c = Case(13, [6], [50], 1, 2, 64, "f16")
    o, lse = c.forward()
    grads = [x.double().cpu().numpy() for x in c.backward(o, lse)]
    rng = np.random.default_rng(0)
    base = [c.q64, c.k64, c.v64]
    for i in range(3):
        u = rng.standard_normal(base[i].shape)
        f = []
        for sign in (1, -1):
            x = [y + sign * 1e-4 * u if j == i else y for j, y in enumerate(base)]
            f.append((co.attend(x[0], x[1].transpose(1, 0, 2), x[2].transpose(1, 0, 2), 64 ** -0.5)[0] * c.g64).sum())
        # the gradient's elements are off by some 2^-10 of themselves, at random signs
        assert abs((f[0] - f[1]) / 2e-4 - (grads[i] * u).sum()) <= 2.0 ** -9 * np.sqrt((grads[i] * u) ** 2).sum() + 1e-3


def test_faults_are_reported_and_bounded():
    c = Case(14, [2, 2], [40, 60], 1, 2, 64, "bf16")
    begin = c.args["kv_begin"]
    for bad in ([0, 40, 1000], [-5, 40, 100], [0, 200, 100]):
        begin.copy_(torch.tensor(bad, dtype=torch.int32))
        o, lse = c.forward()
        c.backward(o, lse)
        torch.cuda.synchronize()
        assert int(c.status) == 2
        c.status.zero_()
    p = Case(15, [2, 2], [40, 60], 1, 2, 64, "bf16", form="padded", pad=60)
    for bad in ([40, 61], [-1, 60]):
        p.args["kv_lens"].copy_(torch.tensor(bad, dtype=torch.int32))
        o, lse = p.forward()
        p.backward(o, lse)
        torch.cuda.synchronize()
        assert int(p.status) == 2
        p.status.zero_()


@pytest.mark.parametrize("n", [2, 100])
def test_captured_calls_replayed(n):
    """A forward and a backward pass in one graph, on new contents and lengths."""
    c = Case(16, [n, n], [90, 140], 2, 2, 128, "bf16", form="padded", pad=140)
    o, lse = c.forward()
    dq = torch.empty_like(c.q)
    dk, dv = torch.empty_like(c.k), torch.empty_like(c.v)
    ws = torch.zeros(R.reskv_cross_attn_workspace(c.T, 4), dtype=torch.uint8, device="cuda")

    def both():
        R.reskv_cross_attn(c.q, c.k, c.v, o, lse=lse, **c.args)
        R.reskv_cross_attn_backward(c.q, c.k, c.v, o, lse, c.g, dq, dk, dv, workspace=ws, **c.args)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        both()
        with pytest.raises(ValueError, match="workspace"):
            with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=s):
                R.reskv_cross_attn_backward(c.q, c.k, c.v, o, lse, c.g, dq, dk, dv, **c.args)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        both()
    c.q.mul_(-0.5)
    c.args["kv_lens"].copy_(torch.tensor([33, 77], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in (o, lse, dq, dk, dv)]
    o2, lse2 = c.forward()
    for x, y in zip(got, (o2, lse2, *c.backward(o2, lse2))):
        assert torch.equal(x, y)
