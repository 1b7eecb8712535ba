"""What an append refuses of its queries before any CUDA call, wherever they would be
turned: in the keys' launch (rows in whole 16-byte words, one type) or in one of their own."""
import pytest

from paper_2607_29591_gb300 import build as B
from paper_2607_29591_gb300 import reskv as R
from test_paged_refusals import P, heads, paged, refused, rotation


@pytest.fixture(scope="module")
def lib():
    B.build()
    return R.load_library()


@pytest.mark.parametrize("kv", [dict(), dict(data=P + 2), dict(dtype=R.RESKV_F32)])     # in the keys' launch; in one of their own
@pytest.mark.parametrize("q,qo,word", [
    (dict(data=None), dict(), "NULL"), (dict(), dict(data=None), "NULL"), (dict(n=0), dict(n=0), "n_heads"), (dict(n=-8), dict(n=-8), "n_heads"),
    (dict(n=65537), dict(n=65537), "n_heads"), (dict(token=-1024), dict(), "strides"), (dict(), dict(head=-128), "strides"),
    (dict(dtype=3), dict(dtype=3), "dtype"), (dict(dtype=-1), dict(dtype=-1), "dtype"), (dict(data=P + 1), dict(), "aligned"),
    (dict(), dict(n=3), "same heads"), (dict(), dict(dtype=R.RESKV_F16), "one dtype")])
def test_queries_of_an_append(lib, kv, q, qo, word):
    k, v = heads(**kv), heads(**kv)
    refused(lib, lib.reskv_paged_append(paged(), 4, P, P, rotation(), k, v, heads(**q), heads(**qo), None), word)


def test_too_many_query_rows(lib):
    n = 1 << 20
    refused(lib, lib.reskv_paged_append(paged(), n, P, P, rotation(), heads(), heads(), heads(n=2048), heads(n=2048), None), "2^31")
