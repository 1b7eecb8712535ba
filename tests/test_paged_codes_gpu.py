"""Codes of groups far from zero, whose bf16 minimum lies a good part of a step below
(or above) the least value: the largest values pass the top code and are held at it,
bit for bit as the definition says, beside values halfway between two codes."""
import numpy as np
import pytest

from test_paged_cache_gpu import append

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("dtype", ["f16", "f32", "bf16"])
@pytest.mark.parametrize("rot,interleaved", [(None, False), (128, False), (128, True)])
def test_codes_of_groups_far_from_zero(dtype, rot, interleaved, group):
    rng = np.random.default_rng(50 + group)
    x = []
    for c in (0.9, 1.3, 40.0, 100.0, 1000.0, -100.0):
        for e in (0.02, 0.05, 0.1):
            x.append(c * (1 + e * rng.random((16, 1, 128))))
    x.append(160 + rng.standard_normal((64, 1, 128)))
    x.append(np.round(8 * (1000 + 4 * rng.standard_normal((64, 1, 128)))) / 8)       # halves in any type
    if dtype != "f16":
        x.append(3e38 * (1 + 0.1 * rng.random((16, 1, 128))))         # scales whose reciprocal is subnormal
    x = np.concatenate(x).astype(np.float32)
    append(rng, 1, 128, group, 64, dtype, (len(x),), (0,), rot=rot, interleaved=interleaved, k=x, v=x[::-1].copy())


def test_a_value_past_the_top_code_beside_halves():
    """1 + 3/1024 twice, 1 + 33/1024 thirty times: scale 2/1024, minimum 1, codes 2, 2, 15, 15, ..."""
    x = np.full((3, 2, 64), 1 + 33 / 1024, np.float32)
    x[0, :, :2] = x[0, :, 32:34] = 1 + 3 / 1024
    x[1, :, 5:7] = x[1, :, 40:42] = 1 + 3 / 1024
    x[2, :, 30:32] = x[2, :, 62:64] = 1 + 3 / 1024
    rng = np.random.default_rng(51)
    for dtype in ("f16", "f32"):
        append(rng, 2, 64, 32, 16, dtype, (3,), (0,), k=x, v=x[:, ::-1].copy())
