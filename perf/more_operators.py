"""Attention over keys that are not a sequence's own, as measurable cases.

Decoder tokens attend to an encoder's states (cross attention, and its gradient),
and sequences that begin with the same tokens attend to one copy of that prefix,
held in 4-bit pages, and to their own tokens behind it.  Shapes are those of the
framework's workloads (8 KV heads, 4 query heads each, head_dim 128; contexts of
4K to 128K; batches of 1 to 64) and smaller or odd ones around them.

op      one pass
cross   tokens of every sequence attend to all of the sequence's states
train   the same, and the gradients of queries, keys and values
shared  every sequence's newest tokens attend to its group's prefix and, causally,
        to its own tokens

States lie as rows [row, head, dim]: equal numbers for every sequence, padded to
one number (``lens`` says how many count) or packed one after another.

The paged cache.  A page holds ``page`` tokens of every KV head, as tiles of 16
tokens: K codes, K scales and minima, V codes, V scales and minima.  A group of
``group`` values x of a row is held as n = rint((x - m) / s) in 0..15, with s =
bf16((max - min) / 15) and m = bf16(min); it stands for s n + m.
"""
import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
DT = {"bf16": torch.bfloat16, "f16": torch.float16}
OUTLIER = 8.0


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _cross(batch, tokens, states, kv=8, per=4, dim=128, dtype="bf16", form="equal", fused=False, empty=False,
           train=False):
    return dict(op="train" if train else "cross", batch=batch, tokens=tokens, states=states, kv=kv, per=per, dim=dim,
                dtype=dtype, form=form, fused=fused, empty=empty)


def _shared(batch, groups, prefix, tail, new=1, kv=8, per=4, dim=128, group=32, page=64, dtype="bf16", ragged=False,
            empty=False):
    return dict(op="shared", batch=batch, groups=groups, prefix=prefix, tail=tail, new=new, kv=kv, per=per, dim=dim,
                group=group, page=page, dtype=dtype, ragged=ragged, empty=empty)


def listed():
    def named(name, case):
        return dict(case, name=name)

    return [
        # one user's decode token against half a minute of encoded sound: launch latency
        named("cross_token", _cross(1, 1, 1500, kv=12, per=1, dim=64)),
        # a decode step of 32 users, documents of unequal length, keys and values out of one projection
        named("cross_step_b32", _cross(32, 1, 6400, form="packed", fused=True)),
        # 16 users' beams of 5, states padded to one length, one user without any; fp16
        named("cross_beams", _cross(16, 5, 1500, kv=16, per=1, dim=64, dtype="f16", form="padded", empty=True)),
        # the prompts of 8 users against encoded pages
        named("cross_prompt", _cross(8, 1024, 4096)),
        # a training step of a toy: captions against a handful of regions
        named("train_small", _cross(2, 77, 50, kv=4, per=2, dim=64, dtype="f16", form="packed", train=True)),
        # captions of 8 images, patches and one summary state
        named("train_images", _cross(8, 512, 577, kv=16, per=1, dim=64, fused=True, train=True)),
        # long answers against long documents, padded
        named("train_long", _cross(4, 2048, 4097, form="padded", train=True)),
        # four answers to one short prompt
        named("shared_few", _shared(4, 1, 2000, 100)),
        # 64 users behind one system prompt
        named("shared_b64", _shared(64, 1, 8192, 512, ragged=True)),
        # four prompts of unequal length, eight answers each, one prompt empty; fp16, groups of 64, small pages
        named("shared_groups", _shared(32, 4, 16384, 300, group=64, page=32, dtype="f16", ragged=True, empty=True)),
        # 16 answers of one prompt, four drafted tokens each to check
        named("shared_drafts", _shared(16, 1, 4096, 700, new=4, ragged=True)),
        # 32 answers about one long document
        named("shared_long", _shared(32, 1, 131072, 1000)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(("cross", "cross", "train", "shared", "shared"))
    per = rng.choice((4, 4, 1, 2, 8, 7))
    kv = rng.choice((8, 8, 16, 4, 2, 1, 3))
    dim = rng.choice((128, 128, 64))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    batch = _log_int(rng, 1, 64)
    heads = kv * per
    if op == "shared":
        groups = min(batch, rng.choice((1, 1, 2, 4, 8)))
        new = 1 if rng.random() < 0.6 else _log_int(rng, 2, 16)
        # no more pairs than the largest case, no more rows held than it holds
        prefix = _log_int(rng, 16, min(131072, (1 << 27) // (batch * heads * new), 1048576 // (groups * kv)))
        tail = _log_int(rng, new, max(new, min(2048, 262144 // (batch * kv))))
        return _shared(batch, groups, prefix, tail, new, kv, per, dim, rng.choice((32, 64, dim)),
                       rng.choice((16, 32, 64, 128)), dtype, rng.random() < 0.6, rng.random() < 0.25)
    tokens = 1 if op == "cross" and rng.random() < 0.5 else _log_int(rng, 2, max(2, min(2048, 65536 // batch)))
    states = _log_int(rng, 1, min(8192, (1 << 30) // (batch * tokens * heads), (1 << 22) // (batch * kv)))
    return _cross(batch, tokens, states, kv, per, dim, dtype, rng.choice(("equal", "padded", "packed")),
                  rng.random() < 0.5, rng.random() < 0.2, op == "train")


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------

def _spread(n, count, part):
    """Numbers up to n, unequal over its upper ``part``."""
    return [max(1, int(n * (1.0 - part * ((i * 0.6180339887498949) % 1.0)))) for i in range(count)]


def _counts(case):
    """Query tokens and states of every sequence."""
    b, form = case["batch"], case["form"]
    q = _spread(case["tokens"], b, 0.5) if form == "packed" else [case["tokens"]] * b
    k = [case["states"]] * b if form == "equal" else _spread(case["states"], b, 0.75)
    if case["empty"] and form != "equal" and b > 1:
        k[-1] = 0
    return q, k


def _members(case):
    """First sequence of every group, and the end."""
    b, g = case["batch"], case["groups"]
    if not case["ragged"]:
        return [i * b // g for i in range(g + 1)]
    at = [0]
    for i in range(g):                                  # later groups are larger
        at.append(at[-1] + max(1, round(2 * (i + 1) * b / (g * (g + 1)))))
    at = [min(x, b - (g - i)) for i, x in enumerate(at)]
    return at[:-1] + [b]


def _held(case):
    """Positions of every group's prefix, and of every sequence's own tokens (its new ones included)."""
    g, b, new = case["groups"], case["batch"], case["new"]
    p = _spread(case["prefix"], g, 0.75) if case["ragged"] else [case["prefix"]] * g
    if case["empty"] and g > 1:
        p[0] = 0
    t = _spread(case["tail"], b, 0.75) if case["ragged"] else [case["tail"]] * b
    return p, [max(new, x) for x in t]


def _row_bytes(dim, group):
    """Bytes of a held K row and V row: 4-bit codes, a bf16 scale and minimum per group."""
    return dim + 2 * 4 * (dim // group)


def work(case):
    d, kv, heads = case["dim"], case["kv"], case["kv"] * case["per"]
    if case["op"] == "shared":
        p, t = _held(case)
        at, n = _members(case), case["new"]
        rows = sum(p) + sum(t)
        pairs = sum(p[g] * n * (at[g + 1] - at[g]) for g in range(case["groups"]))
        pairs += sum(n * x - n * (n - 1) // 2 for x in t)
        return {"bytes": rows * kv * _row_bytes(d, case["group"]) + case["batch"] * n * heads * d * 4,
                "flops": pairs * heads * 4 * d}
    q, k = _counts(case)
    pairs = sum(x * y for x, y in zip(q, k))
    rows = sum(k) if case["form"] != "equal" else case["batch"] * case["states"]
    written = case["batch"] * case["states"] if case["form"] == "padded" else rows
    if case["op"] == "cross":
        return {"bytes": 2 * d * (2 * sum(q) * heads + 2 * rows * kv), "flops": pairs * heads * 4 * d}
    # q, do in, o, dq out; k, v in, dk, dv out
    return {"bytes": 2 * d * (4 * sum(q) * heads + 2 * rows * kv + 2 * written * kv), "flops": pairs * heads * 14 * d}


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
    s, m = ((hi - lo) / 15.0).to(torch.bfloat16), lo.to(torch.bfloat16)
    n = ((y - m.float()) / s.float()).round().clamp(0, 15)
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
    vb = vb.movedim(-2, -4).transpose(-3, -2)                           # [.., r, g, c, tok, 2]
    at = _places(d)[..., None, None, None].expand(vb.shape)
    vb = torch.gather(vb, -4, at)                                       # place p holds chunk p ^ turn
    return torch.cat([kb.flatten(-4), _bytes_of_meta(ks, km).flatten(-2), vb.flatten(-5),
                      _bytes_of_meta(vs, vm).flatten(-2)], -1)


def _unpack(t, d, group):
    """Bytes [.., tile_bytes] of tiles -> float32 values of K and V [.., 16, d]."""
    a, b = 8 * d, 16 * 4 * (d // group)
    kc, kmeta, vc, vmeta = t[..., :a], t[..., a:a + b], t[..., a + b:2 * a + b], t[..., 2 * a + b:]
    kb = kc.unflatten(-1, (16, 4, d // 32, 4)).transpose(-3, -2).flatten(-3)
    vb = vc.unflatten(-1, (8, 8, d // 32, 2, 2))
    at = _places(d)[..., None, None, None].expand(vb.shape)
    vb = torch.gather(vb, -4, at).transpose(-3, -2)                     # [.., r, g, tok, c, 2]
    vb = vb.movedim(-4, -2).flatten(-3).flatten(-3, -2)                 # [.., 16, d/2]

    def values(bytes_, meta):
        n = torch.stack([bytes_ & 15, bytes_ >> 4], -1).flatten(-2).float().unflatten(-1, (-1, group))
        sm = meta.contiguous().view(torch.bfloat16).float().unflatten(-1, (16, 2, d // group))
        return (n * sm[..., 0, :, None] + sm[..., 1, :, None]).flatten(-2)

    return values(kb, kmeta), values(vb, vmeta)


def _values(pages, table, n, d, group):
    """float32 K and V [rows of the table, kv, n, d] of the first n positions; what no page holds is whatever."""
    page = pages.shape[2] * 16
    t = pages[table[:, :-(-n // page)].long().clamp(min=0)]             # [B, np, kv, tiles, bytes]
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


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _ends(counts):
    return [sum(counts[:i]) for i in range(len(counts) + 1)]


def _prepare_cross(case, seed):
    b, kv, per, d = (case[k] for k in ("batch", "kv", "per", "dim"))
    dt, g = DT[case["dtype"]], _gen(seed, 1)
    nq, nk = _counts(case)
    s = dict(case=dict(case), q_begin=None, kv_begin=None, kv_lens=None)
    if case["form"] == "packed":
        s["q_begin"], s["kv_begin"] = _ints(_ends(nq)), _ints(_ends(nk))
    if case["form"] == "padded":
        s["kv_lens"] = _ints(nk)
    rows = sum(nk) if case["form"] == "packed" else b * case["states"]
    first = _ends(nk)[:-1] if case["form"] == "packed" else [i * case["states"] for i in range(b)]
    kvs = torch.cat([_rows(g, kv, rows, d), _rows(g, kv, rows, d)]).transpose(0, 1).to(dt)      # [rows, 2 kv, d]
    s["k"], s["v"] = kvs[:, :kv].contiguous(), kvs[:, kv:].contiguous()
    if case["fused"]:
        both = kvs.contiguous()
        s["k"], s["v"] = both[:, :kv], both[:, kv:]
    # queries akin to one of the states that they see
    seq = torch.arange(b, device=DEV).repeat_interleave(torch.tensor(nq, device=DEV))
    near = torch.zeros((sum(nq), kv, d), device=DEV)
    if rows:
        pick = torch.rand(sum(nq), generator=g, device=DEV) * torch.tensor(nk, device=DEV)[seq]
        pick = (torch.tensor(first, device=DEV)[seq] + pick.long()).clamp(max=rows - 1)
        near = s["k"][pick].float()
    q = 0.3 * near.repeat_interleave(per, 1) + 0.7 * torch.randn((sum(nq), kv * per, d), generator=g, device=DEV)
    s["q"] = q.to(dt).contiguous()
    s["o"] = torch.empty_like(s["q"])
    if case["op"] == "train":
        s["do"] = torch.randn(q.shape, generator=g, device=DEV).to(dt)
        s["lse"] = torch.empty(q.shape[:2], device=DEV)
        s["dq"] = torch.empty_like(s["q"])
        s["dk"], s["dv"] = torch.empty_like(s["k"].contiguous()), torch.empty_like(s["v"].contiguous())
        if case["fused"]:
            both = torch.empty((rows, 2 * kv, d), dtype=dt, device=DEV)
            s["dk"], s["dv"] = both[:, :kv], both[:, kv:]
    return s


def prepare(case, seed):
    if case["op"] != "shared":
        return _prepare_cross(case, seed)
    b, groups, kv, per, d, group, page, n = (case[k] for k in ("batch", "groups", "kv", "per", "dim", "group", "page",
                                                               "new"))
    g = _gen(seed, 2)
    p, t = _held(case)
    at = _members(case)
    need = [-(-x // page) for x in p + t]
    total = sum(need)
    # one pool of pages in shuffled order; what lies behind a last token, and one more page, belongs to nobody
    order = torch.randperm(total + 1, generator=g, device=DEV).to(torch.int32)
    pages = torch.zeros((total + 1, kv, page // 16, _tile_bytes(d, group)), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 26) // (kv * page * d))
    for i in range(0, total, step):
        m = min(step, total - i)
        k, v = (_rows(g, kv, m * page, d).unflatten(1, (m, page // 16, 16)) for _ in range(2))
        pages[order[i:i + m].long()] = _pack(*_codes(k, group), *_codes(v, group)).transpose(0, 1)

    def table(first, counts):
        out, i = torch.full((len(counts), max(1, max(counts))), -1, dtype=torch.int32, device=DEV), first
        for r, c in enumerate(counts):
            out[r, :c] = order[i:i + c]
            i += c
        return out

    s = dict(case=dict(case), pages=pages, prefix_table=table(0, need[:groups]),
             page_table=table(sum(need[:groups]), need[groups:]), prefix_lens=_ints(p), lens=_ints(t),
             seq_begin=_ints(at) if case["ragged"] or b % groups else None)
    # queries akin to a key of their own or of the prefix
    tile = pages[s["page_table"][:, 0].long(), :, 0]                                          # [B, kv, bytes]
    near = _unpack(tile, d, group)[0][:, :, 0]
    if p[-1]:
        far = _unpack(pages[s["prefix_table"][-1:, 0].long(), :, 0], d, group)[0][:, :, 0]
        near = torch.where((torch.arange(b, device=DEV) % 2 == 0)[:, None, None], near, far)
    q = 0.3 * near.repeat_interleave(per, 1)[:, None] + 0.7 * torch.randn((b, n, kv * per, d), generator=g, device=DEV)
    s["q"] = q.flatten(0, 1).to(DT[case["dtype"]]).contiguous()
    s["o"] = torch.empty_like(s["q"])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _padded(begin, lens, rows, batch):
    """Where the rows of [batch, most] lie among ``rows`` packed ones, and which exist."""
    if begin is None:
        first = torch.arange(batch, device=DEV) * (rows // batch)
        have = torch.full((batch,), rows // batch, device=DEV)
    else:
        first, have = begin[:-1].long(), (begin[1:] - begin[:-1]).long()
    seen = have if lens is None else torch.minimum(have, lens.long())
    return first, have, seen


def _plain_cross(s):
    c = s["case"]
    b, kv, per, d = (c[k] for k in ("batch", "kv", "per", "dim"))
    dt = DT[c["dtype"]]
    qf, qn, _ = _padded(s["q_begin"], None, s["q"].shape[0], b)
    kf, kn, seen = _padded(s["kv_begin"], s["kv_lens"], s["k"].shape[0], b)
    tq, tk = torch.arange(c["tokens"], device=DEV), torch.arange(c["states"], device=DEV)
    qi = (qf[:, None] + tq).clamp(max=max(0, s["q"].shape[0] - 1))
    ki = (kf[:, None] + tk).clamp(max=max(0, s["k"].shape[0] - 1))
    see = (tk < seen[:, None])[:, None, None]                                                  # [B, 1, 1, states]
    there = (tq < qn[:, None])[:, :, None, None]

    def of_queries(x):                                                                        # [B, kv, per * tokens, d]
        x = torch.where(there, x[qi].float(), 0.0)
        return x.unflatten(2, (kv, per)).permute(0, 2, 3, 1, 4).flatten(2, 3)

    def back(x):
        x = x.unflatten(2, (per, -1)).permute(0, 3, 1, 2, 4).flatten(2, 3)
        return x[there[:, :, 0, 0]].to(dt)

    def of_states(x):
        return torch.where((tk < seen[:, None])[:, :, None, None], x[ki].float(), 0.0).transpose(1, 2)

    def rows(x, like):                                                                        # [B, kv, states, d] -> packed
        y = torch.zeros(like.shape, device=DEV)
        m = tk < kn[:, None]
        y[ki[m]] = x.transpose(1, 2)[m]
        return y.to(dt)

    q, k, v = of_queries(s["q"]), of_states(s["k"]), of_states(s["v"])
    x = ((q @ k.transpose(-1, -2)) * d ** -0.5).masked_fill_(~see, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    del x
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    o = p @ v
    if c["op"] == "cross":
        return back(o)
    do = of_queries(s["do"])
    dv = p.transpose(-1, -2) @ do
    t = p * (do @ v.transpose(-1, -2) - (do * o).sum(-1, keepdim=True)) * d ** -0.5
    return {"o": back(o), "dq": back(t @ k), "dk": rows(t.transpose(-1, -2) @ q, s["k"]), "dv": rows(dv, s["v"])}


def _plain_shared(s):
    c = s["case"]
    b, n, kv, per, d, group = (c[k] for k in ("batch", "new", "kv", "per", "dim", "group"))
    groups = c["groups"]
    begin = s["seq_begin"].long() if s["seq_begin"] is not None else torch.arange(groups + 1, device=DEV) * (b // groups)
    q = s["q"].float().view(b, n, kv, per, d).permute(0, 2, 3, 1, 4).flatten(2, 3)             # [B, kv, per * n, d]
    # own tokens, causally
    ko, vo = _values(s["pages"], s["page_table"], c["tail"] if c["tail"] > n else n, d, group)
    at = s["lens"].long()[:, None] - n + torch.arange(n, device=DEV)
    see_o = (torch.arange(ko.shape[2], device=DEV) <= at[..., None])[:, None].repeat(1, 1, per, 1)
    xo = ((q @ ko.transpose(-1, -2)) * d ** -0.5).masked_fill(~see_o, -math.inf)
    # the prefix, for a group's sequences at once: slot i of group g is sequence begin[g] + i
    kp, vp = _values(s["pages"], s["prefix_table"], c["prefix"], d, group)
    seq = torch.arange(b, device=DEV)
    group_of = (seq[:, None] >= begin[1:]).sum(-1)
    slot = seq - begin[group_of]
    slots = b                                                                                # no group is larger
    if s["seq_begin"] is None:
        slots = b // groups
    member = (begin[:-1, None] + torch.arange(slots, device=DEV)).clamp(max=b - 1)
    qg = q[member].transpose(1, 2).flatten(2, 3)                                               # [G, kv, slots * per * n, d]
    see_p = torch.arange(kp.shape[2], device=DEV) < s["prefix_lens"][:, None]
    xp = ((qg @ kp.transpose(-1, -2)) * d ** -0.5).masked_fill(~see_p[:, None, None], -math.inf)
    top_p = xp.amax(-1).unflatten(2, (slots, -1)).transpose(1, 2)[group_of, slot]               # [B, kv, per * n]
    top = torch.maximum(xo.amax(-1), top_p)[..., None]
    top = torch.where(top > -math.inf, top, 0.0)
    po = torch.exp(xo - top)
    # each slot's own reference; slots that are no member are dropped again below
    pp = torch.exp(xp - top[member].transpose(1, 2).flatten(2, 3))
    vp = torch.where(see_p[:, None, :, None], vp, 0.0)
    vo = torch.where((torch.arange(vo.shape[2], device=DEV) < s["lens"][:, None])[:, None, :, None], vo, 0.0)
    parts = torch.cat([pp @ vp, pp.sum(-1, keepdim=True)], -1).unflatten(2, (slots, -1)).transpose(1, 2)[group_of, slot]
    both = torch.cat([po @ vo, po.sum(-1, keepdim=True)], -1) + parts
    o = both[..., :d] / torch.where(both[..., d:] > 0, both[..., d:], 1.0)
    return o.unflatten(2, (per, n)).permute(0, 3, 1, 2, 4).reshape(b * n, kv * per, d).to(DT[c["dtype"]])


def run(s):
    c = s["case"]
    if not own:
        return _plain_shared(s) if c["op"] == "shared" else _plain_cross(s)
    from paper_2607_29591_gb300 import reskv as R
    if c["op"] == "shared":
        if "own" not in s:                                # views of the pages, kept with the state as a program keeps them
            s["own"] = R.PagedKV(s["pages"], s["page_table"], c["page"], c["kv"], c["dim"], c["group"])
            s["prefix"] = R.PagedKV(s["pages"], s["prefix_table"], c["page"], c["kv"], c["dim"], c["group"])
        R.reskv_paged_attn_shared(s["own"], s["prefix"], s["q"], s["lens"], s["prefix_lens"], s["o"],
                                  seq_begin=s["seq_begin"])
        return s["o"]
    where = dict(batch=c["batch"], q_begin=s["q_begin"], kv_begin=s["kv_begin"], kv_lens=s["kv_lens"])
    if c["op"] == "cross":
        R.reskv_cross_attn(s["q"], s["k"], s["v"], s["o"], **where)
        return s["o"]
    R.reskv_cross_attn(s["q"], s["k"], s["v"], s["o"], lse=s["lse"], **where)
    R.reskv_cross_attn_backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"], **where)
    return {"o": s["o"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_cross(case, s):
    """Sequence by sequence and KV head by KV head, gradients by automatic differentiation."""
    kv, per, d = case["kv"], case["per"], case["dim"]
    nq, nk = _counts(case)
    train = case["op"] == "train"
    names = ("q", "k", "v") if train else ("q",)
    out = {("o" if not train else "d" + x): torch.zeros(s[x].shape, dtype=torch.float64, device=DEV) for x in names}
    out["o"] = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    q0 = k0 = 0
    for i in range(case["batch"]):
        if case["form"] != "packed":
            k0 = i * case["states"]
        for h in range(kv if nk[i] else 0):
            mine = slice(h * per, (h + 1) * per)
            q = s["q"][q0:q0 + nq[i], mine].double().requires_grad_(train)
            k = s["k"][k0:k0 + nk[i], h].double().requires_grad_(train)
            v = s["v"][k0:k0 + nk[i], h].double().requires_grad_(train)
            o = torch.softmax(torch.einsum("tad,jd->taj", q, k) / math.sqrt(d), -1) @ v
            out["o"][q0:q0 + nq[i], mine] = o.detach()
            if train:
                o.backward(s["do"][q0:q0 + nq[i], mine].double())
                out["dq"][q0:q0 + nq[i], mine] = q.grad
                out["dk"][k0:k0 + nk[i], h] = k.grad
                out["dv"][k0:k0 + nk[i], h] = v.grad
        q0, k0 = q0 + nq[i], k0 + nk[i]
    return out if train else out["o"]


def _exact_rows(s, table, n, values):
    """[kv, n, d] K (values 0) or V (values 1) of the first n positions of one row of a page table, by the address
    of every value."""
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
    tile = table.long()[t // page] * (kv * (page // 16)) + (t % page) // 16                     # of head 0
    flat = s["pages"].view(-1)
    k = torch.arange(d // group, device=DEV)

    def half(at):                                       # a bf16 is the upper half of a float32
        bits = (flat[at].int() << 16) | (flat[at + 1].int() << 24)
        return bits.view(torch.float32).double().repeat_interleave(group, -1)

    out = torch.empty((kv, n, d), dtype=torch.float64, device=DEV)
    for h in range(kv):
        start = (tile + h * (page // 16)) * _tile_bytes(d, group) + section
        n4 = (flat[start + byte] >> (4 * (x % 2)).to(torch.uint8)) & 15
        at = start + 8 * d + row * meta + 2 * k
        out[h] = n4.double() * half(at) + half(at + 2 * (d // group))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] != "shared":
        return _exact_cross(case, s)
    kv, per, d, n = case["kv"], case["per"], case["dim"], case["new"]
    p, t = _held(case)
    at = _members(case)
    out = torch.zeros((case["batch"], n, kv * per, d), dtype=torch.float64, device=DEV)
    q = s["q"].double().view(case["batch"], n, kv, per, d)
    for g in range(case["groups"]):
        kp, vp = (_exact_rows(s, s["prefix_table"][g], p[g], i) for i in range(2))
        for i in range(at[g], at[g + 1]):
            ko, vo = (_exact_rows(s, s["page_table"][i], t[i], j) for j in range(2))
            # a row's newest token sees all, the one before it all but one, ...
            see = torch.ones((n, p[g] + t[i]), dtype=torch.bool, device=DEV).tril(p[g] + t[i] - n)
            for h in range(kv):
                k, v = torch.cat([kp[h], ko[h]]), torch.cat([vp[h], vo[h]])
                x = torch.einsum("nad,td->ant", q[i, :, h], k) / math.sqrt(d)
                w = torch.softmax(x.masked_fill(~see, -math.inf), -1)
                out[i, :, h * per:(h + 1) * per] = torch.einsum("ant,td->nad", w, v)
    return out.view(-1, kv * per, d)
