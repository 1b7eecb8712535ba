"""What cross attention and its gradient refuse, before any CUDA call (no GPU needed; the
pointers are never followed), and the layout of their struct."""
import ctypes
import os
import struct
import subprocess

import pytest
import torch

from paper_2607_29591_gb300 import build as B
from paper_2607_29591_gb300 import reskv as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                              # a 256-byte aligned address


@pytest.fixture(scope="module")
def lib():
    B.build()
    return R.load_library()


def test_struct_layout_matches_c(lib, tmp_path):
    s = R.reskv_cross_attn_args
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "reskv.h"', "int main(void){",
             f'printf("%zu\\n", sizeof({s.__name__}));']
    lines += [f'printf("%zu\\n", offsetof({s.__name__}, {f}));' for f, _ in s._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]
    packed = R._pack_cross.__self__
    assert packed.size == ctypes.sizeof(s) == struct.calcsize(packed.format)


def heads(data=P, token=1024, head=128, n=8, dtype=R.RESKV_BF16):
    return R.reskv_heads(data, token, head, n, dtype)


def args(**over):
    f = dict(q=heads(n=32), k=heads(), v=heads(), o=heads(n=32), lse=P, q_begin=P, kv_begin=P, kv_lens=P, n_tokens=10,
             n_rows=100, batch=3, head_dim=128, scale=0.0, status=None, workspace=P, workspace_bytes=1 << 20)
    f.update(over)
    return R.reskv_cross_attn_args(**f)


REFUSED = [
    (dict(q=heads(data=None, n=32)), "q is NULL"), (dict(o=heads(data=None, n=32)), "o is NULL"), (dict(k=heads(data=None)), "k is NULL"),
    (dict(v=heads(data=None)), "v is NULL"), (dict(head_dim=96), "head_dim"), (dict(q=heads(n=32, dtype=R.RESKV_F32)), "bf16 or fp16"),
    (dict(k=heads(dtype=R.RESKV_F16)), "dtype"), (dict(o=heads(n=32, dtype=R.RESKV_F16)), "dtype"), (dict(o=heads(n=31)), "same heads"),
    (dict(v=heads(n=4)), "same heads"), (dict(q=heads(n=33), o=heads(n=33)), "multiple"), (dict(q=heads(n=520), o=heads(n=520)), "64"),
    (dict(batch=0), "batch"), (dict(batch=(1 << 24) + 1), "batch"), (dict(n_tokens=-1), "n_tokens"), (dict(n_tokens=1 << 26), "n_tokens"),
    (dict(n_rows=-1), "n_rows"), (dict(n_rows=1 << 28), "n_rows"), (dict(q_begin=None), "without q_begin"),
    (dict(kv_begin=None), "without kv_begin"), (dict(lse=P + 2), "aligned"), (dict(kv_lens=P + 1), "aligned"),
    (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale"), (dict(q=heads(data=P + 1, n=32)), "aligned"),
    (dict(k=heads(token=-1)), "strides"), (dict(q=heads(n=0), o=heads(n=0)), "n_heads")]


@pytest.mark.parametrize("over,word", REFUSED)
def test_refusals(lib, over, word):
    a = args(**over)
    g = [heads(n=32), heads(n=32), heads(), heads()]
    for st in (lib.reskv_cross_attn(a, None), lib.reskv_cross_attn_backward(a, *g, None)):
        assert st == R.RESKV_ERR_INVALID_ARG and word in R.reskv_last_error(), R.reskv_last_error()


@pytest.mark.parametrize("over,at,grad,word", [
    (dict(lse=None), 0, heads(n=32), "lse"), (dict(workspace=None), 0, heads(n=32), "workspace"),
    (dict(workspace=P + 128), 0, heads(n=32), "workspace"), (dict(workspace_bytes=1023), 0, heads(n=32), "workspace"),
    (dict(), 0, heads(n=8), "d_o and d_q"), (dict(), 1, heads(n=32, dtype=R.RESKV_F16), "d_o and d_q"), (dict(), 2, heads(n=4), "d_k and d_v"),
    (dict(), 3, heads(dtype=R.RESKV_F32), "d_k and d_v"), (dict(), 0, heads(data=None, n=32), "d_o is NULL"),
    (dict(), 1, heads(data=P + 1, n=32), "aligned"), (dict(), 2, heads(data=None), "d_k is NULL"), (dict(), 3, heads(head=-1), "strides")])
def test_backward_refusals(lib, over, at, grad, word):
    g = [heads(n=32), heads(n=32), heads(), heads()]
    g[at] = grad
    st = lib.reskv_cross_attn_backward(args(**over), *g, None)
    assert st == R.RESKV_ERR_INVALID_ARG and word in R.reskv_last_error(), R.reskv_last_error()


def test_missing_arguments(lib):
    assert lib.reskv_cross_attn(None, None) == R.RESKV_ERR_INVALID_ARG
    assert lib.reskv_cross_attn_backward(args(), None, heads(n=32), heads(), heads(), None) == R.RESKV_ERR_INVALID_ARG
    assert lib.reskv_cross_attn_workspace(None) == 0 and R.reskv_cross_attn_workspace(10, 32) >= 1024 + 10 * 32 * 4
    assert lib.reskv_cross_attn(args(n_tokens=0, q=heads(data=None, n=32), o=heads(data=None, n=32)), None) == R.RESKV_OK


def test_tensors_are_looked_over():
    t = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        R.reskv_cross_attn(t, t, t, t)
    with pytest.raises(ValueError, match="tokens, heads, dim"):
        R.reskv_cross_attn(t[0], t, t, t)
