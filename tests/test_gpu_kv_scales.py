"""Scales of the scores at the ends of their range: what the kernels cannot multiply by
is refused."""

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv4_util import Batch4, values64
from kv_util import BF, Batch

pytestmark = pytest.mark.gpu
LARGEST = 2.0 ** 127  # (the factor with log2 e ends at 1.38 times it)


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("new,lens", [([1, 1], [300, 33]), ([40, 3], [300, 33])])
@pytest.mark.parametrize("four,exp", [(True, 0), (True, 20), (True, -20), (False, 0)])
def test_the_largest_scales(four, exp, new, lens):
    """Large ones are taken, with queries as small; refused where the factor with log2 e is no number."""
    b = (Batch4 if four else Batch)(new, lens, 8, 2, 64, 16, BF).fill()
    if four:
        b.caches[0] = b.caches[0]._replace(exp=exp)
        b.keys = [values64(*h, exp) for h in b.held[0]]
    caches = b.caches if four else (b.k_cache, b.v_cache)
    b.q = b.q * 2.0 ** -110  # (products of 2^-16 of the largest are normal numbers still)
    scale = 2.0 ** (109 - max(exp, 0))
    kv = b.handle()
    out, lse = kv.paged_attention(b.q, *caches, scale=scale, want_lse=True)
    kv.check()
    if exp >= 0:
        for bad in (1.5 * LARGEST * 2.0 ** -exp, 1.9 * LARGEST * 2.0 ** -exp, 0.0, -1.0, float("nan"), float("inf")):
            with pytest.raises(pkg.SmetricError):
                kv.paged_attention(b.q, *caches, scale=bad)
    kv.check()
    kv.close()
    b.assert_attends(out, lse, scale)
