"""Operators around a full (not yet compressed) KV cache, as measurable cases.

A layer's queries and keys are rotated by their positions, its keys and values
go into a paged cache held in 4 bits, its queries attend over that cache, and a
prompt's rows are read back for compression.  Shapes are those of the
framework's workloads (LLaMA-3.1-8B attention: 8 KV heads, 4 query heads each,
head_dim 128; contexts of 4K to 128K; batches of 1 to 64) and smaller or odd ones
around them.

op      one pass
rope    rotation of q and k (or, backward, of their gradients)
append  rotation of q and k, 4-bit rows of k and v into pages, and the read of the
        rows just written, as values (what a prompt's compression reads next)
attn    attention of every sequence's newest tokens over its pages
gather  the values of a whole prompt out of the pages, as rows for compression

The paged cache.  A page holds ``page`` tokens of every KV head, as tiles of 16
tokens: K codes, K scales and minima, V codes, V scales and minima.  A group of
``group`` values x of a row is held as n = rint((x - m) / s) in 0..15, with s =
bf16((max - min) / 15) and m = bf16(min); it stands for s n + m.
"""
import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
OUTLIER = 8.0


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _rope(tokens, heads, kv, dim=128, rot=128, dtype="bf16", interleaved=False, backward=False,
          fused=False, factor=1.0, reach=131072):
    return dict(op="rope", tokens=tokens, heads=heads, kv=kv, dim=dim, rot=rot, dtype=dtype,
                interleaved=interleaved, backward=backward, fused=fused, factor=factor, reach=reach)


def _append(batch, new, kv=8, per=4, dim=128, rot=128, group=32, page=64, dtype="bf16", start=0,
            interleaved=False, padding=False):
    return dict(op="append", batch=batch, new=new, kv=kv, per=per, dim=dim, rot=rot, group=group, page=page,
                dtype=dtype, start=start, interleaved=interleaved, padding=padding)


def _attn(batch, length, new=1, kv=8, per=4, dim=128, group=32, page=64, dtype="bf16", ragged=False,
          window=0, empty=False):
    return dict(op="attn", batch=batch, length=length, new=new, kv=kv, per=per, dim=dim, group=group, page=page,
                dtype=dtype, ragged=ragged, window=window, empty=empty)


def _gather(batch, length, kv=8, dim=128, group=32, page=64, dtype="bf16", ragged=False):
    return dict(op="gather", batch=batch, length=length, kv=kv, dim=dim, group=group, page=page, dtype=dtype,
                ragged=ragged)


def listed():
    def named(name, case):
        return dict(case, name=name)

    return [
        # one user's decode token, a layer's q and k: launch latency
        named("rope_token", _rope(1, 32, 8)),
        # a prompt chunk out of a fused q, k, v projection, positions scaled by 4 for a long context
        named("rope_prompt", _rope(8191, 32, 8, fused=True, factor=4.0)),
        # the gradient of a training batch in 32 bits: adjacent pairs, half of the head rotated
        named("rope_grad", _rope(16384, 32, 8, rot=64, dtype="f32", interleaved=True, backward=True)),
        # a decode step of 8 users, each token behind a context of its own
        named("append_step_b8", _append(8, 1, start=32000)),
        # a small model's short prompts: 64-wide heads, part of the head rotated, padded to one length
        named("append_ragged", _append(3, 333, kv=4, per=2, dim=64, rot=32, group=64, page=16, dtype="f16",
                                       interleaved=True, padding=True)),
        # the prompts of 8 users at once, the benchmark's context
        named("append_prompt", _append(8, 4096)),
        # one user, a short conversation: latency
        named("attn_token_1k", _attn(1, 1000)),
        # the benchmark's batch and context, before compression
        named("attn_step_32k_b8", _attn(8, 32768)),
        # many users with conversations of unequal length, one of them new; fp16, groups of 64
        named("attn_step_b64", _attn(64, 8192, group=64, page=32, dtype="f16", ragged=True, empty=True)),
        # a chunk of a prompt behind the chunks before it
        named("attn_chunk", _attn(2, 8192, new=512)),
        # one user's prompt to compress
        named("gather_4k", _gather(1, 4096)),
        # the benchmark's batch, prompts of unequal length
        named("gather_32k_b8", _gather(8, 32768, ragged=True)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rope", "append", "append", "attn", "attn", "attn", "gather"))
    per = rng.choice((4, 4, 2, 1, 8, 7))
    dim = rng.choice((128, 128, 64))
    group = rng.choice((32, 64, dim))
    page = rng.choice((16, 32, 64, 128))
    kv = rng.choice((8, 8, 4, 2, 1, 3))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    if op == "rope":
        dim = rng.choice((128, 128, 64, 96, 256))
        return _rope(_log_int(rng, 1, 16384), kv * per, kv, dim, rng.choice((dim, dim // 2)),
                     rng.choice(("bf16", "f16", "f32")), rng.random() < 0.5, rng.random() < 0.3,
                     rng.random() < 0.5, rng.choice((1.0, 4.0, 8.0)), rng.choice((4096, 32768, 131072)))
    if op == "append":
        batch = _log_int(rng, 1, 64)
        new = 1 if rng.random() < 0.4 else _log_int(rng, 1, max(1, 262144 // (batch * kv)))
        return _append(batch, new, kv, per, dim, rng.choice((dim, dim // 2)), group, page, dtype,
                       _log_int(rng, 1, 32768), rng.random() < 0.5, rng.random() < 0.3)
    if op == "gather":
        batch = _log_int(rng, 1, 16)
        return _gather(batch, _log_int(rng, 16, max(16, min(131072, 2097152 // (batch * kv)))), kv, dim, group,
                       page, rng.choice(("bf16", "f16")), rng.random() < 0.5)
    batch = _log_int(rng, 1, 64)
    length = _log_int(rng, 16, max(16, min(131072, 2097152 // (batch * kv))))
    new = 1 if rng.random() < 0.6 else _log_int(rng, 2, 16)
    if rng.random() < 0.15:
        new = min(_log_int(rng, 16, 512), max(1, (1 << 27) // (batch * kv * per * length)))
    return _attn(batch, length, min(new, length), kv, per, dim, group, page, dtype, rng.random() < 0.5,
                 rng.choice((0, 0, 0, 128, 1000)), rng.random() < 0.2)


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------

def _row_bytes(dim, group):
    """Bytes of a K row and a V row: 4-bit codes, a bf16 scale and minimum per group."""
    return dim + 2 * 4 * (dim // group)


def _lengths(case):
    """Tokens of every sequence: the case's, or spread over its upper three quarters; one may be empty."""
    b, n = case["batch"], case["length"]
    lens = [n] * b
    if case.get("ragged"):
        lens = [max(1, min(n, int(n * (1.0 - 0.75 * ((i * 0.6180339887498949) % 1.0))))) for i in range(b)]
    if case.get("empty") and len(lens) > 1:
        lens[-1] = 0
    return lens


def _new_lengths(case):
    """Tokens appended to every sequence: with padding, sequence i leaves its last 7 i tokens out."""
    return [max(1, case["new"] - 7 * i) if case["padding"] else case["new"] for i in range(case["batch"])]


def work(case):
    d = case["dim"]
    if case["op"] == "rope":
        rows = case["tokens"] * (case["heads"] + case["kv"])
        return {"bytes": rows * d * 2 * SIZE[case["dtype"]] + case["tokens"] * (case["rot"] * 4 + 4),
                "flops": rows * case["rot"] * 3}
    if case["op"] == "append":
        tokens, size = sum(_new_lengths(case)), SIZE[case["dtype"]]
        q, kv = tokens * case["kv"] * case["per"], tokens * case["kv"]
        # q in and out; k and v in, their 4-bit rows out, the rows' values out
        return {"bytes": q * d * 2 * size + kv * (2 * d * size + _row_bytes(d, case["group"]) + 2 * d * size),
                "flops": (q + kv) * case["rot"] * 3 + kv * 2 * d * 6}
    lens = _lengths(case)
    if case["op"] == "gather":
        rows = case["batch"] * case["length"] * case["kv"]
        return {"bytes": sum(lens) * case["kv"] * _row_bytes(d, case["group"]) + rows * 2 * d * SIZE[case["dtype"]],
                "flops": sum(lens) * case["kv"] * 2 * d * 2}
    n, w, heads = case["new"], case["window"], case["kv"] * case["per"]
    seen = pairs = 0
    for length in lens:
        first = max(0, length - n)
        seen += length - (max(0, first - w + 1) if w else 0)
        for p in range(max(0, length - n), length):
            pairs += min(p + 1, w) if w else p + 1
    return {"bytes": seen * case["kv"] * _row_bytes(d, case["group"])
            + case["batch"] * n * heads * d * 2 * SIZE[case["dtype"]],
            "flops": pairs * heads * 4 * d}


# ---------------------------------------------------------------------------
# the paged cache in plain operations
# ---------------------------------------------------------------------------

def _tile_bytes(dim, group):
    return 16 * _row_bytes(dim, group)


def _places(dim):
    """places[r, g]: the place of chunk g in pair row r of a tile's V codes."""
    r, g = torch.arange(8, device=DEV)[:, None], torch.arange(8, device=DEV)[None]
    return g ^ (2 * (r % 4) if dim == 128 else 4 * ((r >> 1) & 1))


def _codes(x, group):
    """Codes [.., d] and scales, minima [.., d / group] of float32 rows x [.., d]."""
    y = x.unflatten(-1, (-1, group))
    lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    s = ((hi - lo) / torch.full_like(hi, 15.0)).to(torch.bfloat16)      # by a tensor: a correctly rounded quotient
    m = lo.to(torch.bfloat16)
    s = torch.where(s.float() < 2.0 ** -126, torch.zeros_like(s), s)
    n = ((y - m.float()) / s.float()).round().clamp(0, 15)
    n = torch.where(s.float() == 0, torch.zeros_like(n), n)
    return n.flatten(-2).to(torch.uint8), s.squeeze(-1), m.squeeze(-1)


def _bytes_of_meta(s, m):
    return torch.cat([s, m], -1).contiguous().view(torch.uint8)


def _pack(kn, ks, km, vn, vs, vm):
    """Tiles [.., 16, ..] of K and V codes, scales and minima -> bytes [.., tile_bytes]."""
    d = kn.shape[-1]
    kb = kn[..., 0::2] | (kn[..., 1::2] << 4)                           # [.., 16, d/2]
    kb = kb.unflatten(-1, (d // 32, 4, 4)).transpose(-3, -2)            # [.., 16, t, c, 4]
    vb = vn[..., 0::2] | (vn[..., 1::2] << 4)
    vb = vb.unflatten(-1, (d // 32, 8, 2)).unflatten(-4, (8, 2))        # [.., r, tok, c, g, 2]
    vb = vb.movedim(-2, -4)                                             # [.., r, g, tok, c, 2]
    vb = vb.transpose(-3, -2)                                           # [.., r, g, c, tok, 2]
    at = _places(d)[..., None, None, None].expand(8, 8, *vb.shape[-3:])
    vb = torch.gather(vb, -4, at.expand(vb.shape))                      # place p holds chunk p ^ swz
    return torch.cat([kb.flatten(-4), _bytes_of_meta(ks, km).flatten(-2), vb.flatten(-5),
                      _bytes_of_meta(vs, vm).flatten(-2)], -1)


def _unpack(t, d, group):
    """Bytes [.., tile_bytes] of tiles -> float32 values of K and V [.., 16, d]."""
    a, b = 8 * d, 16 * 4 * (d // group)
    kc, kmeta, vc, vmeta = t[..., :a], t[..., a:a + b], t[..., a + b:2 * a + b], t[..., 2 * a + b:]
    kb = kc.unflatten(-1, (16, 4, d // 32, 4)).transpose(-3, -2).flatten(-3)
    vb = vc.unflatten(-1, (8, 8, d // 32, 2, 2))
    at = _places(d)[..., None, None, None].expand(8, 8, *vb.shape[-3:])
    vb = torch.gather(vb, -4, at.expand(vb.shape)).transpose(-3, -2)    # [.., r, g, tok, c, 2]
    vb = vb.movedim(-4, -2).flatten(-3).flatten(-3, -2)                 # [.., 16, d/2]

    def values(bytes_, meta):
        n = torch.stack([bytes_ & 15, bytes_ >> 4], -1).flatten(-2).float().unflatten(-1, (-1, group))
        sm = meta.contiguous().view(torch.bfloat16).float().unflatten(-1, (16, 2, d // group))
        return (n * sm[..., 0, :, None] + sm[..., 1, :, None]).flatten(-2)

    return values(kb, kmeta), values(vb, vmeta)


def _values(pages, table, n, d, group):
    """float32 K and V [batch, kv, n, d] of every sequence's first n positions."""
    page = pages.shape[2] * 16
    t = pages[table[:, :-(-n // page)].long()]                          # [B, np, kv, tiles, bytes]
    k, v = _unpack(t.transpose(1, 2), d, group)
    return k.flatten(2, 4)[:, :, :n], v.flatten(2, 4)[:, :, :n]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed, tag):
    return torch.Generator(device=DEV).manual_seed(1000003 * (int(seed) % (1 << 40)) + tag)


def _rows(g, heads, tokens, d):
    """[heads, tokens, d]: normal values, in every head four channels 8 times larger."""
    x = torch.randn((heads, tokens, d), generator=g, device=DEV)
    c = torch.randint(0, d // 4, (heads, 1), generator=g, device=DEV) + torch.arange(0, d, d // 4, device=DEV)
    return x * torch.ones(heads, d, device=DEV).scatter_(1, c, OUTLIER)[:, None]


def _table(n, rot, factor):
    """[n, rot / 2, 2] cos and sin of position / factor at base 500000, in 64 bits rounded to 32."""
    f = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot) / factor
    a = torch.arange(n, dtype=torch.float64, device=DEV)[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float()


def _paged(case, seed, span, fill):
    """Pages in shuffled order for ``span`` positions of every sequence, the first ``fill`` of each written; the
    last page belongs to none."""
    b, kv, d, group, page = (case[k] for k in ("batch", "kv", "dim", "group", "page"))
    per = -(-span // page)
    g = _gen(seed, 3)
    table = torch.randperm(b * per, generator=g, device=DEV).view(b, per).to(torch.int32)
    pages = torch.zeros((b * per + 1, kv, page // 16, _tile_bytes(d, group)), dtype=torch.uint8, device=DEV)
    if fill:
        used = -(-fill // page)
        for i in range(b):
            k = _rows(g, kv, used * page, d).unflatten(1, (used, page // 16, 16))
            v = _rows(g, kv, used * page, d).unflatten(1, (used, page // 16, 16))
            pages[table[i, :used].long()] = _pack(*_codes(k, group), *_codes(v, group)).transpose(0, 1)
    return pages, table


def prepare(case, seed):
    op, d = case["op"], case["dim"]
    dt = DT[case["dtype"]]
    g = _gen(seed, 1)
    s = dict(case=dict(case))
    if op == "rope":
        n, h, kv = case["tokens"], case["heads"], case["kv"]
        x = _rows(g, h + kv, n, d).transpose(0, 1).to(dt)
        # a fused projection's rows also hold v, which is not rotated
        x = torch.cat([x, x[:, :kv]], 1).contiguous() if case["fused"] else x.contiguous()
        s["q"], s["k"] = x[:, :h], x[:, h:h + kv]
        if not case["fused"]:
            s["q"], s["k"] = s["q"].contiguous(), s["k"].contiguous()
        s["q_out"] = torch.empty((n, h, d), dtype=dt, device=DEV)
        s["k_out"] = torch.empty((n, kv, d), dtype=dt, device=DEV)
        s["table"] = _table(case["reach"], case["rot"], case["factor"])
        first = torch.randint(0, max(1, case["reach"] - n), (1,), generator=g, device=DEV)
        s["positions"] = ((first + torch.arange(n, device=DEV)) % case["reach"]).to(torch.int32)
    elif op == "append":
        b, n, kv, heads = case["batch"], case["new"], case["kv"], case["kv"] * case["per"]
        span = case["start"] + n
        s["pages"], s["page_table"] = _paged(case, seed, span, 0)
        for name, h in (("q", heads), ("k", kv), ("v", kv)):
            s[name] = _rows(g, h, b * n, d).transpose(0, 1).to(dt).contiguous()
        s["q_out"] = torch.zeros_like(s["q"])
        s["k_out"] = torch.empty((b, kv, n, d), dtype=dt, device=DEV)
        s["v_out"] = torch.empty((b, kv, n, d), dtype=dt, device=DEV)
        s["table"] = _table(span, case["rot"], 1.0)
        # contexts of their own: sequence i starts 5 i positions earlier
        start = (case["start"] - 5 * torch.arange(b, device=DEV)).clamp(min=0)
        new = torch.tensor(_new_lengths(case), device=DEV)
        i = torch.arange(n, device=DEV)
        pos = torch.where(i < new[:, None], start[:, None] + i, -1)
        s["positions"] = pos.flatten().to(torch.int32)
        s["seqs"] = torch.arange(b, device=DEV).repeat_interleave(n).to(torch.int32)
        s["starts"], s["lens"] = start.to(torch.int32), (start + new).to(torch.int32)
    else:
        lens = _lengths(case)
        s["pages"], s["page_table"] = _paged(case, seed, case["length"], case["length"])
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        if op == "attn":
            b, n, heads = case["batch"], case["new"], case["kv"] * case["per"]
            # peaked queries: part of a cached key, as the framework's workloads draw them
            at = torch.randint(0, case["length"], (b,), generator=g, device=DEV)
            at = torch.minimum(at, (s["lens"] - 1).clamp(min=0))
            tile = s["pages"][s["page_table"][torch.arange(b, device=DEV), at // case["page"]].long()]
            k, _ = _unpack(tile, d, case["group"])
            near = k.flatten(2, 3)[torch.arange(b, device=DEV), :, at % case["page"]]      # [B, kv, d]
            near = near.repeat_interleave(case["per"], 1)[:, None] * 0.3
            q = near + 0.7 * torch.randn((b, n, heads, d), generator=g, device=DEV)
            s["q"] = q.flatten(0, 1).to(dt).contiguous()
            s["o"] = torch.empty_like(s["q"])
        else:
            shape = (case["batch"], case["kv"], case["length"], d)
            s["k_out"] = torch.empty(shape, dtype=dt, device=DEV)
            s["v_out"] = torch.empty(shape, dtype=dt, device=DEV)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _rotate(x, cs, rot, interleaved, backward):
    """Rows x [T, H, d] in float32 turned by cs [T, rot / 2, 2]."""
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    s = -s if backward else s
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    ya, yb = a * c - b * s, b * c + a * s
    y = torch.stack([ya, yb], -1).flatten(-2) if interleaved else torch.cat([ya, yb], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_append(s):
    c = s["case"]
    d, group, page, b, n, kv = (c[k] for k in ("dim", "group", "page", "batch", "new", "kv"))
    pos, live = s["positions"].long(), s["positions"] >= 0
    cs = s["table"][pos.clamp(min=0)]
    dt = DT[c["dtype"]]
    q = _rotate(s["q"].float(), cs, c["rot"], c["interleaved"], False).to(dt)
    q = torch.where(live[:, None, None], q, s["q"])
    kn, ks, km = _codes(_rotate(s["k"].float(), cs, c["rot"], c["interleaved"], False), group)
    vn, vs, vm = _codes(s["v"].float(), group)

    def values(x, sc, m):
        y = x.float().unflatten(-1, (-1, group)) * sc.float()[..., None] + m.float()[..., None]
        y = torch.where(live[:, None, None], y.flatten(-2), 0.0)
        return y.view(b, n, kv, d).transpose(1, 2).to(dt)

    # the same rows into their tiles, byte by byte; what is padding goes into the page that belongs to none
    at = s["page_table"][s["seqs"].long(), pos.clamp(min=0) // page].long()
    at = torch.where(live, at, s["pages"].shape[0] - 1)
    slot = pos.clamp(min=0) % page
    tile, row = slot // 16, slot % 16
    w = torch.arange(d // 2, device=DEV)
    u, i = w // 4, w % 4
    k_at = row[:, None] * (d // 2) + ((u % 4) * (d // 32) + u // 4) * 4 + i
    u, i = w // 2, w % 2
    r = (row // 2)[:, None]
    v_at = r * d + _places(d)[r, u % 8] * (d // 8) + (u // 8) * 4 + (row % 2)[:, None] * 2 + i
    meta = 4 * (d // group)
    m_at = row[:, None] * meta + torch.arange(meta, device=DEV)
    base = 8 * d + 16 * meta
    where = torch.cat([k_at, 8 * d + m_at, base + v_at, base + 8 * d + m_at], 1)
    data = torch.cat([kn[..., 0::2] | (kn[..., 1::2] << 4), _bytes_of_meta(ks, km),
                      vn[..., 0::2] | (vn[..., 1::2] << 4), _bytes_of_meta(vs, vm)], -1)
    heads = torch.arange(kv, device=DEV)
    flat = (((at[:, None] * kv + heads) * (page // 16) + tile[:, None])[..., None] * _tile_bytes(d, group)
            + where[:, None])
    s["pages"].view(-1)[flat] = data
    return {"q": q, "k": values(kn, ks, km), "v": values(vn, vs, vm)}


def _visible(s, length):
    """[B, new, length]: whether query i of a sequence sees position t."""
    n, w = s["case"]["new"], s["case"]["window"]
    at = s["lens"].long()[:, None] - n + torch.arange(n, device=s["lens"].device)
    t = torch.arange(length, device=s["lens"].device)
    see = t <= at[..., None]
    return see & (t > at[..., None] - w) if w else see


def _plain_attn(s):
    c = s["case"]
    b, n, kv, per, d = (c[k] for k in ("batch", "new", "kv", "per", "dim"))
    k, v = _values(s["pages"], s["page_table"], c["length"], d, c["group"])
    q = s["q"].float().view(b, n, kv, per, d).permute(0, 2, 3, 1, 4).reshape(b, kv, per * n, d)
    x = (q @ k.transpose(-1, -2)) * d ** -0.5
    see = _visible(s, c["length"])[:, None].repeat(1, 1, per, 1)
    top = x.masked_fill(~see, -math.inf).amax(-1, keepdim=True)
    p = torch.where(see, torch.exp(x - torch.where(see.any(-1, keepdim=True), top, 0.0)), 0.0)
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(total > 0, total, 1.0)
    return o.view(b, kv, per, n, d).permute(0, 3, 1, 2, 4).reshape(b * n, kv * per, d).to(DT[c["dtype"]])


def _plain_gather(s):
    c = s["case"]
    k, v = _values(s["pages"], s["page_table"], c["length"], c["dim"], c["group"])
    live = (torch.arange(c["length"], device=DEV) < s["lens"][:, None])[:, None, :, None]
    return {"k": torch.where(live, k, 0.0).to(DT[c["dtype"]]), "v": torch.where(live, v, 0.0).to(DT[c["dtype"]])}


def _handle(s):
    """The framework's view of the state's pages, kept with the state as a program keeps it."""
    if "handle" not in s:
        from paper_2607_29591_gb300 import reskv as R
        c = s["case"]
        s["handle"] = R.PagedKV(s["pages"], s["page_table"], c["page"], c["kv"], c["dim"], c["group"])
    return s["handle"]


def run(s):
    c = s["case"]
    if not own:
        if c["op"] == "rope":
            cs = s["table"][s["positions"].long()]
            dt = DT[c["dtype"]]
            return {x: _rotate(s[x].float(), cs, c["rot"], c["interleaved"], c["backward"]).to(dt) for x in "qk"}
        return {"append": _plain_append, "attn": _plain_attn, "gather": _plain_gather}[c["op"]](s)
    from paper_2607_29591_gb300 import reskv as R
    if c["op"] == "rope":
        R.reskv_rope(s["q"], s["q_out"], s["positions"], s["table"], k=s["k"], k_out=s["k_out"],
                     interleaved=c["interleaved"], backward=c["backward"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["op"] == "append":
        R.reskv_paged_append(_handle(s), s["k"], s["v"], s["seqs"], s["positions"], table=s["table"],
                             interleaved=c["interleaved"], q=s["q"], q_out=s["q_out"])
        R.reskv_paged_gather(_handle(s), s["lens"], s["k_out"], s["v_out"], starts=s["starts"])
        return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
    if c["op"] == "attn":
        R.reskv_paged_attn(_handle(s), s["q"], s["lens"], s["o"], window=c["window"])
        return s["o"]
    R.reskv_paged_gather(_handle(s), s["lens"], s["k_out"], s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_turned(x, table, positions, rot, interleaved, sign):
    """Complex multiplication of every pair by its position's cos + i sin."""
    out = x.double().clone()
    z = torch.view_as_complex(table.double())[positions][:, None]
    z = z.conj() if sign < 0 else z
    if interleaved:
        y = torch.view_as_complex(out[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * z
        out[..., :rot] = torch.view_as_real(y).flatten(-2)
    else:
        y = torch.complex(out[..., :rot // 2], out[..., rot // 2:rot]) * z
        out[..., :rot // 2], out[..., rot // 2:rot] = y.real, y.imag
    return out


def _exact_held(x, group):
    """What a row is held as, its codes chosen in 64 bits."""
    y = x.unflatten(-1, (-1, group))
    low = y.amin(-1, keepdim=True)
    s = ((y.amax(-1, keepdim=True) - low) / 15).to(torch.bfloat16).double()
    m = low.to(torch.bfloat16).double()
    return (torch.clamp(torch.round((y - m) / s), 0, 15) * s + m).flatten(-2)


def _exact_rows(s, seq, n, values):
    """[kv, n, d] K (values 0) or V (values 1) of a sequence's first n positions, by the address of every value."""
    c = s["case"]
    d, group, page, kv = c["dim"], c["group"], c["page"], c["kv"]
    t, x = torch.arange(n, device=DEV)[:, None], torch.arange(d, device=DEV)[None]
    row, meta = t % 16, 4 * (d // group)
    section = values * (8 * d + 16 * meta)
    if values == 0:
        unit = x // 8
        byte = row * (d // 2) + (unit % 4) * (d // 8) + (unit // 4) * 4 + (x % 8) // 2
    else:
        pair, g = row // 2, (x // 4) % 8
        turn = (pair % 4) * 2 if d == 128 else (pair // 2 % 2) * 4
        byte = pair * d + (g ^ turn) * (d // 8) + (x // 32) * 4 + (row % 2) * 2 + (x % 4) // 2
    tile = s["page_table"][seq].long()[t // page] * (kv * (page // 16)) + (t % page) // 16     # of head 0
    flat = s["pages"].view(-1)
    head = torch.arange(kv, device=DEV)[:, None, None] * (page // 16)
    start = (tile + head) * _tile_bytes(d, group) + section
    n4 = (flat[start + byte] >> (4 * (x % 2)).to(torch.uint8)) & 15
    k = torch.arange(d // group, device=DEV)
    at = start + 8 * d + row * meta + 2 * k

    def half(at):                                       # a bf16 is the upper half of a float32
        bits = (flat[at].int() << 16) | (flat[at + 1].int() << 24)
        return bits.view(torch.float32).double().repeat_interleave(group, -1)

    return n4.double() * half(at) + half(at + 2 * (d // group))


def exact(case, seed):
    s = prepare(case, seed)
    d = case["dim"]
    if case["op"] == "rope":
        sign = -1 if case["backward"] else 1
        return {x: _exact_turned(s[x], s["table"], s["positions"].long(), case["rot"], case["interleaved"], sign)
                for x in "qk"}
    if case["op"] == "append":
        live = (s["positions"] >= 0)[:, None, None]
        pos = s["positions"].long().clamp(min=0)
        turned = {x: _exact_turned(s[x], s["table"], pos, case["rot"], case["interleaved"], 1) for x in "qk"}

        def rows(x):
            y = torch.where(live, _exact_held(x, case["group"]), 0.0)
            return y.view(case["batch"], case["new"], case["kv"], d).transpose(1, 2).contiguous()

        return {"q": torch.where(live, turned["q"], s["q"].double()), "k": rows(turned["k"]),
                "v": rows(s["v"].double())}
    lens = _lengths(case)
    if case["op"] == "gather":
        out = {x: torch.zeros((case["batch"], case["kv"], case["length"], d), dtype=torch.float64, device=DEV)
               for x in "kv"}
        for i, n in enumerate(lens):
            for j, x in enumerate("kv"):
                out[x][i, :, :n] = _exact_rows(s, i, n, j)
        return out
    n, per, kv = case["new"], case["per"], case["kv"]
    out = torch.zeros((case["batch"], n, kv * per, d), dtype=torch.float64, device=DEV)
    q = s["q"].double().view(case["batch"], n, kv, per, d)
    for i, length in enumerate(lens):
        if length == 0:
            continue
        see = _visible(s, length)[i]
        k, v = _exact_rows(s, i, length, 0), _exact_rows(s, i, length, 1)
        for h in range(kv):
            x = torch.einsum("nad,td->ant", q[i, :, h], k[h]) / math.sqrt(d)
            x = x.masked_fill(~see, -math.inf)
            p = torch.nan_to_num(torch.softmax(x, -1), nan=0.0)
            out[i, :, h * per:(h + 1) * per] = torch.einsum("ant,td->nad", p, v[h])
    return out.view(-1, kv * per, d)
