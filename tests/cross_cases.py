"""Cross attention's gradients against fp64 by their norms, one sequence and KV head at a time."""
import numpy as np

from oracle import cross_oracle as co
from paged_cases import HALF_ULP

LEAST = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25}        # half a smallest step


def check_norms(c):
    """c: a test_cross_gpu.Case.  Runs it forward and backward."""
    scale = c.d ** -0.5 if c.scale is None else c.scale
    dq, dk, dv = (x.double().cpu().numpy() for x in c.backward(*c.forward()))
    for b, (t, r, _) in enumerate(c.sequences()):
        ref, tol = co.gradient_norms(c.q64[t], c.k64[r].transpose(1, 0, 2), c.v64[r].transpose(1, 0, 2), c.g64[t], scale,
                                     HALF_ULP[c.dtype], LEAST[c.dtype])
        n = t.stop - t.start
        heads = lambda x: x.reshape(n, c.kv, c.per, c.d).transpose(1, 0, 2, 3)  # noqa: E731
        for i, (name, got, want) in enumerate((("dq", heads(dq[t]), heads(ref[0])), ("dk", dk[r].transpose(1, 0, 2), ref[1]),
                                               ("dv", dv[r].transpose(1, 0, 2), ref[2]))):
            for h in range(c.kv):
                off = np.linalg.norm(got[h] - want[h])
                assert off <= tol[i, h], (name, b, h, off, tol[i, h], np.linalg.norm(want[h]))
