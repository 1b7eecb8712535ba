"""Building paged 4-bit caches for tests: random rows, their held form, pages in
shuffled order whose unused slots are garbage (all ones: codes 15, NaN scales)."""
import numpy as np
import torch

from oracle import paged_oracle as po
from paper_2607_29591_gb300 import reskv as R

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}      # of |x|: p significant bits, 2^-p


def rows(rng, shape, d):
    """Normal values with a few channels 8 times larger."""
    x = rng.standard_normal(shape + (d,)).astype(np.float32)
    x[..., rng.integers(0, d, 3)] *= 8
    return x


def paged(rng, lens, kv, d, group, page, extra_pages=2, table_pages=None):
    """A PagedKV of random held rows and their fp64 values [kv, len, d] per sequence."""
    need = [-(-n // page) for n in lens]
    per = max(max(need), 1) if table_pages is None else table_pages
    total = sum(need) + extra_pages
    order = rng.permutation(total)
    table = np.full((len(lens), per), -7, np.int32)              # unused entries are out of range
    pages = np.full((total, kv, R.reskv_paged_head_bytes(page, d, group)), 0xFF, np.uint8)
    at, values = 0, []
    for b, n in enumerate(lens):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        held = [po.hold(rows(rng, (kv, n), d), group) for _ in range(2)]
        for h in range(kv):
            for t in range(n):
                for which in range(2):
                    c, s, m = (a[h, t] for a in held[which])
                    po.put_row(pages[table[b, t // page]], h, t % page, d, group, which, c, s, m)
        values.append([po.held_value(*held[i]) for i in range(2)])
    kvc = R.PagedKV(torch.from_numpy(pages).cuda(), torch.from_numpy(table).cuda(), page, kv, d, group)
    return kvc, values, pages, table


def as_type(x, dtype):
    """numpy -> CUDA tensor of the dtype, and the fp64 values it then has."""
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(DT[dtype])
    return t.cuda(), t.double().numpy()
