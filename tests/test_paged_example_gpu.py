"""The example that runs rotation, pages, attention, reading back, construction and
compressed decode together (examples/prompt_then_compress.py)."""
import importlib.util
import os

import pytest
import torch

from paper_2607_29591_gb300 import reskv as R

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "prompt_then_compress.py")


def test_prompt_then_compress():
    spec = importlib.util.spec_from_file_location("prompt_then_compress", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.main(batch=2, prompt=700, chunk=256, steps=3, budget=700, page_tokens=32)
    assert r["page_bytes"] * 3 < r["bf16_bytes"]
    assert torch.isfinite(r["paged"]).all() and torch.isfinite(r["compressed"]).all()
    # With a budget of the whole prompt nothing is evicted: the compressed cache then holds the pages' values
    # (rounded to bf16 on the way: 2^-8 of every key and value, and of the paged output).  A logit is off by at most
    # 2^-8 of scale sum |q k|, an output by that twice and 2^-7 more of the largest value.
    K = r["K"].float().abs().amax()
    V = r["V"].float().abs().amax()
    q = r["last_q"].float().abs()
    logit = float((q.sum(-1).max() * K) * 128 ** -0.5)
    bound = (2 * 2.0 ** -8 * logit + 2.0 ** -7) * float(V)
    assert float((r["paged"] - r["compressed"]).abs().max()) <= bound
    # and far nearer than that on average: roundings do not add up
    assert r["off"] < 0.02
    small = m.main(batch=1, prompt=512, chunk=512, steps=2, budget=128, page_tokens=16)
    assert torch.isfinite(small["compressed"]).all() and small["off"] < 1.0
    R.reskv_test_inject(R.RESKV_TEST_FAIL_ALLOC, 0)
