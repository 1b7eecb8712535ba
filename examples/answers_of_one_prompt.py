"""Several answers to one prompt about one document: a decoder layer whose tokens attend to the prompt, which all
answers share in 4-bit pages, to their own tokens behind it, and to the document's encoded states; then the
gradient that would train the attention to the states.

    python examples/answers_of_one_prompt.py

Every step is the call that a serving or training loop makes: rotation and append in one launch,
reskv_paged_attn_shared over the prompt's pages and the answers' own, reskv_cross_attn to the states (the answers
are one sequence there: they read the same ones), reskv_cross_attn_backward.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_29591_gb300 import reskv as R  # noqa: E402

H_KV, G, D = 8, 4, 128
H = H_KV * G


def main(answers=16, prompt=1000, steps=6, states=577, page_tokens=32, seed=0):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)

    def rows(n, heads):
        return torch.randn((n, heads, D), generator=g, device=dev).bfloat16()

    table = R.reskv_rope_table(R.reskv_rope_config_default(), prompt + steps)
    per_prompt, per_answer = -(-prompt // page_tokens), -(-steps // page_tokens)
    pages = R.reskv_paged_pages(per_prompt + answers * per_answer, H_KV, page_tokens)
    order = torch.randperm(pages.shape[0], generator=g, device=dev).to(torch.int32)
    prefix = R.PagedKV(pages, order[:per_prompt][None].contiguous(), page_tokens, H_KV)
    own = R.PagedKV(pages, order[per_prompt:].view(answers, per_answer).contiguous(), page_tokens, H_KV)

    # the prompt, once for all answers
    k, v = rows(prompt, H_KV), rows(prompt, H_KV)
    R.reskv_paged_append(prefix, k, v, torch.zeros(prompt, dtype=torch.int32, device=dev),
                         torch.arange(prompt, dtype=torch.int32, device=dev), table=table)
    # the document's states, keys and values out of one projection
    both = torch.randn((states, 2 * H_KV, D), generator=g, device=dev).bfloat16()
    state_k, state_v = both[:, :H_KV], both[:, H_KV:]

    prompt_len = torch.tensor([prompt], dtype=torch.int32, device=dev)
    seqs = torch.arange(answers, dtype=torch.int32, device=dev)
    taken = []
    for i in range(steps):
        q, k, v = rows(answers, H), rows(answers, H_KV), rows(answers, H_KV)
        # positions go on behind the prompt, places among the own pages begin at 0
        at = torch.full((answers,), prompt + i, dtype=torch.int32, device=dev)
        R.reskv_rope(q, q, at, table, k=k, k_out=k)
        R.reskv_paged_append(own, k, v, seqs, at - prompt)
        o = torch.empty_like(q)
        R.reskv_paged_attn_shared(own, prefix, q, at - prompt + 1, prompt_len, o)
        # what it found asks the document
        found = torch.empty_like(o)
        lse = torch.empty((answers, H), device=dev)
        R.reskv_cross_attn(o, state_k, state_v, found, lse=lse)
        taken.append(dict(q=q, o=o, found=found, lse=lse))
    own.check_status()
    prefix.check_status()

    # the last step's gradient of sum(found * d) with respect to the queries and the states
    last = taken[-1]
    d = torch.randn(last["found"].shape, generator=g, device=dev).bfloat16()
    d_q, d_both = torch.empty_like(d), torch.empty_like(both)
    R.reskv_cross_attn_backward(last["o"], state_k, state_v, last["found"], last["lse"], d, d_q, d_both[:, :H_KV], d_both[:, H_KV:])
    return dict(steps=taken, d=d, d_q=d_q, d_both=d_both, both=both, own=own, prefix=prefix, prompt=prompt)


if __name__ == "__main__":
    r = main()
    print(f"{len(r['steps'])} tokens of {r['steps'][0]['q'].shape[0]} answers; |d_q| {r['d_q'].float().norm():.3f}, "
          f"|d_states| {r['d_both'].float().norm():.3f}")
