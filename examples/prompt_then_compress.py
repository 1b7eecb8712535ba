"""One attention layer from prompt to compressed decode: a prompt goes through in
chunks, its keys and values into 4-bit pages; some tokens are decoded from the
pages; then the pages are read back, compressed to a budget, and decoding goes on
from the compressed cache.

    python examples/prompt_then_compress.py

The layer has LLaMA-3.1-8B's attention shape and made-up weights.  Every step is the
call that a serving loop makes: rotation and append of a chunk in one launch,
attention of the chunk (or token) over the pages, reskv_paged_gather into
reskv_build_cache, reskv_append and reskv_decode_attn.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_29591_gb300 import reskv as R  # noqa: E402

H_KV, G, D, WIDTH = 8, 4, 128, 4096
H = H_KV * G


def main(batch=2, prompt=2048, chunk=512, steps=8, budget=1024, page_tokens=64, seed=0):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    # random weights, queries akin to the keys; tokens of 32 topics, so that attention has something to find
    w_k, w_v = (torch.randn((WIDTH, H_KV, D), generator=g, device=dev) * WIDTH ** -0.5 for _ in range(2))
    w_q = 0.5 * w_k.repeat_interleave(G, 1) + 0.3 * WIDTH ** -0.5 * torch.randn((WIDTH, H, D), generator=g, device=dev)
    w_qkv = torch.cat([w_q, w_k, w_v], 1).view(WIDTH, (H + 2 * H_KV) * D).bfloat16()
    topic = torch.randint(0, 32, (batch, prompt + steps), generator=g, device=dev)
    hidden = torch.randn((32, WIDTH), generator=g, device=dev)[topic]
    hidden = (hidden + 0.5 * torch.randn(hidden.shape, generator=g, device=dev)).bfloat16()

    # positions scaled for four times the context that the frequencies are made for
    cfg = R.reskv_rope_config_default(scaling=R.RESKV_ROPE_WAVELENGTH, factor=4.0, original_positions=8192.0)
    table = R.reskv_rope_table(cfg, prompt + steps)

    # pages handed out in any order: here, dealt at random
    per = -(-(prompt + steps) // page_tokens)
    pages = R.reskv_paged_pages(batch * per, H_KV, page_tokens)
    order = torch.randperm(batch * per, generator=g, device=dev).to(torch.int32).view(batch, per)
    kv = R.PagedKV(pages, order, page_tokens, H_KV)

    def layer(first, n):
        """Tokens first .. first + n - 1 of every sequence: append, then attend over all so far."""
        qkv = (hidden[:, first:first + n].reshape(batch * n, WIDTH) @ w_qkv).view(batch * n, H + 2 * H_KV, D)
        q, k, v = qkv[:, :H], qkv[:, H:H + H_KV], qkv[:, H + H_KV:]
        seqs = torch.arange(batch, dtype=torch.int32, device=dev).repeat_interleave(n)
        pos = (first + torch.arange(n, dtype=torch.int32, device=dev)).repeat(batch)
        R.reskv_paged_append(kv, k, v, seqs, pos, table=table, q=q, q_out=q)
        lens = torch.full((batch,), first + n, dtype=torch.int32, device=dev)
        out = torch.empty((batch * n, H, D), dtype=torch.bfloat16, device=dev)
        R.reskv_paged_attn(kv, q, lens, out)
        return q, out

    for first in range(0, prompt, chunk):
        q, out = layer(first, min(chunk, prompt - first))
    observed = q.view(batch, -1, H, D)[:, -128:].transpose(1, 2).contiguous()     # the prompt's last queries
    decoded = [layer(prompt + i, 1) for i in range(steps)]
    kv.check_status()

    # the prompt's rows as a layer's input of the construction
    K, V = (torch.empty((batch, H_KV, prompt, D), dtype=torch.bfloat16, device=dev) for _ in range(2))
    R.reskv_paged_gather(kv, torch.full((batch,), prompt, dtype=torch.int32, device=dev), K, V)
    cache = R.reskv_build_cache(R.reskv_config_default(batch=batch, n_layers=1, n_kv_heads=H_KV, group=G, seq_len=prompt,
                                                       budget=budget, n_obs=128, append_capacity=steps), [K], [V], [observed])
    new = torch.empty((2, batch, H_KV, 1, D), dtype=torch.bfloat16, device=dev)
    compressed = []
    for i, (q, _) in enumerate(decoded):
        # the token's held key and value join the compressed cache, as they joined the pages
        at = torch.full((batch,), prompt + i, dtype=torch.int32, device=dev)
        R.reskv_paged_gather(kv, at + 1, new[0], new[1], starts=at)
        R.reskv_append(cache, 0, new[0].squeeze(2), new[1].squeeze(2))
        o = torch.empty((batch, H, D), dtype=torch.float32, device=dev)
        R.reskv_decode_attn(cache, 0, q.contiguous(), o)
        compressed.append(o)
    R.reskv_check_status(cache)
    paged = torch.stack([o.view(batch, H, D).float() for _, o in decoded])
    small = torch.stack(compressed)
    cache.free()
    held = pages.numel()
    result = dict(K=K, V=V, last_q=decoded[-1][0], paged=paged, compressed=small,
                  page_bytes=held, bf16_bytes=2 * batch * H_KV * per * page_tokens * D * 2,
                  off=float((small - paged).norm() / paged.norm()))
    return result


if __name__ == "__main__":
    r = main()
    print(f"pages hold {r['page_bytes'] / 1e6:.1f} MB, bf16 rows would take {r['bf16_bytes'] / 1e6:.1f} MB")
    print(f"decode from the compressed cache against decode from all pages: relative L2 {r['off']:.3f}")
    assert np.isfinite(r["off"])
