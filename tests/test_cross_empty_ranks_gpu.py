"""Cross attention and its gradient where a cluster has more CTAs than a sequence has tiles: batches padded to
thousands of rows whose sequences are far shorter, so that some of a cluster's CTAs see no states (or, with
few tokens beside many, no rows) and the row's sums are those of the others."""
import pytest

from cross_cases import check_norms
from test_cross_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f16")])
@pytest.mark.parametrize("n", [1, 3, 20, 100])
@pytest.mark.parametrize("lens", [[4000, 100, 1, 0], [129, 128, 3000, 1000]])
def test_short_sequences_in_a_long_padding(lens, n, d, dtype):
    c = Case(41 + n, [n] * 4, lens, 1, 4, d, dtype, form="padded", pad=4096)
    c.check()
    for _ in range(3):
        check_norms(c)


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f16")])
@pytest.mark.parametrize("counts,lens", [([900, 1, 40], [50, 60, 70]), ([1, 1, 700], [2000, 3, 130])])
def test_few_tokens_beside_many(counts, lens, d, dtype):
    c = Case(43, counts, lens, 1, 4, d, dtype)
    c.check()
    check_norms(c)
