"""The operators over keys that are not a sequence's own, run together as a decoder layer has them."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import cross_oracle as co
from paged_cases import HALF_ULP
from paper_2607_29591_gb300 import reskv as R

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def held(kv, n):
    """fp64 K and V [batch, heads, n, d] of what the pages hold (fp32 values: one rounding of s n + m)."""
    out = [torch.empty((kv.batch, kv.n_kv_heads, n, kv.head_dim), device="cuda") for _ in range(2)]
    R.reskv_paged_gather(kv, torch.full((kv.batch,), n, dtype=torch.int32, device="cuda"), *out)
    return [x.double().cpu().numpy() for x in out]


def test_a_layer_of_answers():
    import answers_of_one_prompt as ex
    answers, prompt, steps = 7, 150, 3
    r = ex.main(answers=answers, prompt=prompt, steps=steps, states=200)
    scale, unit = ex.D ** -0.5, HALF_ULP["bf16"]
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    pk, pv = held(r["prefix"], prompt)
    ok, ov = held(r["own"], steps)
    sk, sv = f64(r["both"][:, :ex.H_KV]).transpose(1, 0, 2), f64(r["both"][:, ex.H_KV:]).transpose(1, 0, 2)
    for i, s in enumerate(r["steps"]):
        q, o, found = f64(s["q"]), f64(s["o"]), f64(s["found"])
        for b in range(answers):
            k, v = np.concatenate([pk[0], ok[b][:, :i + 1]], 1), np.concatenate([pv[0], ov[b][:, :i + 1]], 1)
            ro, _, xm, vm = co.attend(q[b:b + 1], k, v, scale)
            # weights and held values of 11 bits, logits and sums in fp32, the output's rounding
            tol = ((2 * ex.D * 2.0 ** -23 * xm + 2.0 ** -10 + 2.0 ** -16) * vm)[..., None] + unit * np.abs(ro) * 1.01
            assert (np.abs(o[b:b + 1] - ro) <= tol).all()
        ro, _, xm, vm = co.attend(o, sk, sv, scale)
        tol = ((2 * ex.D * 2.0 ** -23 * xm + unit + 2.0 ** -16) * vm)[..., None] + unit * np.abs(ro) * 1.01
        assert (np.abs(found - ro) <= tol).all()
    last = r["steps"][-1]
    ref, tol = co.gradient(f64(last["o"]), sk, sv, f64(r["d"]), scale, unit, 2.0 ** -134)
    d_both = f64(r["d_both"]).transpose(1, 0, 2)
    for got, want, off in ((f64(r["d_q"]), ref[0], tol[0]), (d_both[:ex.H_KV], ref[1], tol[1]), (d_both[ex.H_KV:], ref[2], tol[2])):
        assert (np.abs(got - want) <= off * 1.01).all()


def test_one_workspace_for_all_and_two_streams():
    """A workspace of the largest size serves all the calls in turn; two streams run them at once, each with its own."""
    import answers_of_one_prompt as ex
    want = ex.main(answers=20, prompt=700, steps=2)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(ex.main(answers=20, prompt=700, steps=2))
    torch.cuda.synchronize()
    for r in got:
        for a, b in zip(want["steps"], r["steps"]):
            assert all(torch.equal(a[x], b[x]) for x in a)
        assert torch.equal(want["d_q"], r["d_q"]) and torch.equal(want["d_both"], r["d_both"])
    # one buffer: the paged call's tickets stay zero behind the gradient
    kv, prefix = want["own"], want["prefix"]
    T, H = 20, ex.H
    size = max(R.reskv_paged_attn_shared_workspace(kv, prefix, T, H), R.reskv_paged_attn_workspace(kv, T, H), R.reskv_cross_attn_workspace(T, H))
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    s = want["steps"][-1]
    both = want["both"]
    lens, plen = torch.full((T,), 2, dtype=torch.int32, device="cuda"), torch.tensor([700], dtype=torch.int32, device="cuda")
    for _ in range(3):
        d_q, d_both = torch.empty_like(s["o"]), torch.empty_like(both)
        R.reskv_cross_attn_backward(s["o"], both[:, :ex.H_KV], both[:, ex.H_KV:], s["found"], s["lse"], want["d"], d_q,
                                    d_both[:, :ex.H_KV], d_both[:, ex.H_KV:], workspace=ws)
        o, plain = torch.empty_like(s["o"]), torch.empty_like(s["o"])
        R.reskv_paged_attn(kv, s["q"], lens, plain, workspace=ws)
        R.reskv_paged_attn_shared(kv, prefix, s["q"], lens, plen, o, workspace=ws)
        assert torch.equal(o, s["o"]) and torch.equal(d_q, want["d_q"]) and torch.equal(d_both, want["d_both"])
        assert int(ws[:1024].to(torch.int32).sum()) == 0
