"""What the rotation, the paged cache and its attention refuse, before any CUDA
call (no GPU needed; the pointers are never followed), and the layout of their
structs."""
import ctypes
import os
import subprocess

import pytest

from paper_2607_29591_gb300 import build as B
from paper_2607_29591_gb300 import reskv as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                              # a 16-byte aligned address


@pytest.fixture(scope="module")
def lib():
    B.build()
    return R.load_library()


def test_struct_layouts_match_c(lib, tmp_path):
    structs = [R.reskv_heads, R.reskv_rotation, R.reskv_rope_config, R.reskv_paged_kv, R.reskv_rows, R.reskv_paged_attn_args]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "reskv.h"', "int main(void){"]
    for s in structs:
        lines.append(f'printf("%zu\\n", sizeof({s.__name__}));')
        lines += [f'printf("%zu\\n", offsetof({s.__name__}, {f}));' for f, _ in s._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for s in structs:
        want += [ctypes.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]
    assert got == want


def test_packed_structs_have_the_structs_sizes():
    import struct
    for f, s in (("Pqqii", R.reskv_heads), ("Pqii", R.reskv_rotation), ("Pqqqi4x", R.reskv_rows), ("PqqiiPqqiiPPPqfiPQ", R.reskv_paged_attn_args)):
        assert struct.calcsize(f) == ctypes.sizeof(s)


def refused(lib, status, word, st=R.RESKV_ERR_INVALID_ARG):
    assert status == st and word in R.reskv_last_error(), (status, R.reskv_last_error())


def heads(data=P, token=1024, head=128, n=8, dtype=R.RESKV_BF16):
    return R.reskv_heads(data, token, head, n, dtype)


def rotation(table=P, n=100, rot=128, interleaved=0):
    return R.reskv_rotation(table, n, rot, interleaved)


def paged(**over):
    f = dict(pages=P, n_pages=10, page_table=P, batch=2, table_pages=5, page_tokens=64, n_kv_heads=8, head_dim=128,
             quant_group=32, status=None)
    f.update(over)
    return R.reskv_paged_kv(**f)


def test_head_bytes(lib):
    assert lib.reskv_paged_head_bytes(16, 128, 32) == 2560 and lib.reskv_paged_head_bytes(64, 64, 64) == 4 * 1152
    for bad in ((0, 128, 32), (24, 128, 32), (2048, 128, 32), (64, 96, 32), (64, 128, 16), (64, 64, 128), (-16, 128, 32)):
        assert lib.reskv_paged_head_bytes(*bad) == 0
    with pytest.raises(ValueError):
        R.reskv_paged_head_bytes(24, 128, 32)


@pytest.mark.parametrize("over,word", [
    (dict(pos=None), "NULL"), (dict(n=3), "n_tensors"), (dict(d=7), "head_dim"), (dict(d=514), "head_dim"), (dict(tokens=-1), "n_tokens"),
    (dict(tokens=1 << 30), "n_tokens"), (dict(rot=rotation(table=None)), "table"), (dict(rot=rotation(table=P + 4)), "aligned"),
    (dict(rot=rotation(rot=130)), "rot_dim"), (dict(rot=rotation(rot=3)), "rot_dim"), (dict(rot=rotation(n=0)), "n_positions"),
    (dict(rot=rotation(interleaved=2)), "interleaved"), (dict(x=heads(data=None)), "NULL"), (dict(x=heads(data=P + 1)), "aligned"),
    (dict(x=heads(dtype=3)), "dtype"), (dict(y=heads(n=7)), "same heads"), (dict(y=heads(dtype=R.RESKV_F16)), "dtype"),
    (dict(x=heads(n=0), y=heads(n=0)), "n_heads"), (dict(x=heads(token=-1)), "strides")])
def test_rope_refusals(lib, over, word):
    a = dict(rot=rotation(), pos=P, tokens=4, d=128, n=1, x=heads(), y=heads())
    a.update(over)
    refused(lib, lib.reskv_rope(a["rot"], a["pos"], a["tokens"], a["d"], a["n"], a["x"], a["y"], 0, None, None), word)


@pytest.mark.parametrize("over,word", [
    (dict(rot_dim=3), "rot_dim"), (dict(rot_dim=514), "rot_dim"), (dict(base=1.0), "base"), (dict(factor=0.5), "factor"),
    (dict(factor=float("nan")), "factor"), (dict(scaling=5), "scaling"), (dict(scaling=-1), "scaling"), (dict(magnitude=-1.0), "magnitude"),
    (dict(scaling=R.RESKV_ROPE_BASE, rot_dim=2), "rot_dim"), (dict(scaling=R.RESKV_ROPE_WAVELENGTH, low_freq=4.0), "low_freq"),
    (dict(scaling=R.RESKV_ROPE_YARN, beta_slow=64.0), "beta"), (dict(scaling=R.RESKV_ROPE_YARN, original_positions=0.0), "original")])
def test_rope_table_refusals(lib, over, word):
    cfg = R.reskv_rope_config_default(**over)
    refused(lib, lib.reskv_rope_table(cfg, 16, P, None), word)


def test_rope_table_arguments(lib):
    cfg = R.reskv_rope_config_default()
    refused(lib, lib.reskv_rope_table(cfg, 0, P, None), "n_positions")
    refused(lib, lib.reskv_rope_table(cfg, 5, None, None), "NULL")
    refused(lib, lib.reskv_rope_table(cfg, 5, P + 4, None), "aligned")


CACHE = [(dict(pages=None), "pages"), (dict(pages=P + 8), "aligned"), (dict(page_table=None), "page_table"), (dict(page_tokens=24), "page_tokens"),
         (dict(head_dim=96), "head_dim"), (dict(quant_group=16), "quant_group"), (dict(n_pages=0), "n_pages"), (dict(n_kv_heads=0), "n_kv_heads"),
         (dict(batch=0), "batch"), (dict(table_pages=1 << 26), "2^31")]


@pytest.mark.parametrize("over,word", CACHE)
def test_cache_refusals(lib, over, word):
    kv = paged(**over)
    refused(lib, lib.reskv_paged_append(kv, 4, P, P, rotation(), heads(), heads(), None, None, None), word)
    refused(lib, lib.reskv_paged_gather(kv, None, P, 4, R.reskv_rows(P, 0, 0, 0, 0), None, None), word)
    a = R.reskv_paged_attn_args(q=heads(n=32), o=heads(n=32), lens=P, n_tokens=4, workspace=P, workspace_bytes=1 << 30)
    refused(lib, lib.reskv_paged_attn(kv, a, None), word)


@pytest.mark.parametrize("over,word", [
    (dict(k=heads(n=4)), "n_kv_heads"), (dict(v=heads(dtype=R.RESKV_F32)), "dtype"), (dict(k=heads(data=None)), "NULL"),
    (dict(seqs=None), "NULL"), (dict(pos=None), "NULL"), (dict(q=heads()), "together"), (dict(q=heads(), qo=heads(), rot=None), "rotation"),
    (dict(tokens=-1), "n_tokens"), (dict(rot=rotation(rot=256)), "rot_dim"), (dict(q=heads(), qo=heads(n=3)), "same heads")])
def test_append_refusals(lib, over, word):
    a = dict(tokens=4, seqs=P, pos=P, rot=rotation(), k=heads(), v=heads(), q=None, qo=None)
    a.update(over)
    refused(lib, lib.reskv_paged_append(paged(), a["tokens"], a["seqs"], a["pos"], a["rot"], a["k"], a["v"], a["q"], a["qo"], None), word)


def test_gather_refusals(lib):
    row = R.reskv_rows(P, 0, 0, 0, R.RESKV_BF16)
    refused(lib, lib.reskv_paged_gather(paged(), None, None, 4, row, row, None), "lens")
    refused(lib, lib.reskv_paged_gather(paged(), None, P, 4, None, None, None), "NULL")
    refused(lib, lib.reskv_paged_gather(paged(), None, P, -1, row, row, None), "n must")
    refused(lib, lib.reskv_paged_gather(paged(), None, P, 4, row, R.reskv_rows(P, 0, 0, 0, R.RESKV_F16), None), "dtype")
    refused(lib, lib.reskv_paged_gather(paged(), None, P, 4, R.reskv_rows(P + 1, 0, 0, 0, 0), None, None), "aligned")
    refused(lib, lib.reskv_paged_gather(paged(), None, P, 4, R.reskv_rows(P, -8, 0, 0, 0), None, None), "strides")


@pytest.mark.parametrize("over,word", [
    (dict(q=heads(n=12), o=heads(n=12)), "multiple"), (dict(q=heads(n=1024), o=heads(n=1024)), "64 per"), (dict(o=heads(n=16)), "same heads"),
    (dict(q=heads(n=32, dtype=R.RESKV_F32)), "bf16 or fp16"), (dict(o=heads(n=32, dtype=R.RESKV_F16)), "q's dtype"), (dict(lens=None), "lens"),
    (dict(n_tokens=-2), "n_tokens"), (dict(n_tokens=3), "multiple of batch"), (dict(scale=float("inf")), "scale"), (dict(window=-1), "window"),
    (dict(n_tokens=1 << 28), "2^31"), (dict(workspace=None), "workspace"), (dict(workspace=P + 16), "workspace"),
    (dict(workspace_bytes=1), "workspace"), (dict(q=heads(n=32, data=P + 1)), "aligned"), (dict(lse=P + 2), "lse")])
def test_attn_refusals(lib, over, word):
    f = dict(q=heads(n=32), o=heads(n=32), lens=P, n_tokens=4, workspace=P, workspace_bytes=1 << 30)
    f.update(over)
    refused(lib, lib.reskv_paged_attn(paged(), R.reskv_paged_attn_args(**f), None), word)
    refused(lib, lib.reskv_paged_attn(paged(), None, None), "NULL")


def test_binding_checks_tensors_before_the_call(lib):
    import torch
    x = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        R.reskv_rope(x, x, torch.zeros(4, dtype=torch.int32), torch.zeros((9, 64, 2)))
    with pytest.raises(ValueError, match="together"):
        R.reskv_rope(x, x, torch.zeros(4, dtype=torch.int32), torch.zeros((9, 64, 2)), k=x)
    with pytest.raises(ValueError, match="q must be"):
        R.reskv_rope(x[0], x[0], torch.zeros(4, dtype=torch.int32), torch.zeros((9, 64, 2)))
    with pytest.raises(ValueError, match="pages"):
        R.PagedKV(torch.zeros(100, dtype=torch.uint8), torch.zeros((1, 1), dtype=torch.int32), 64, 8)
