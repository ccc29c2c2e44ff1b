"""Page numbers that no page has: keys and values behind them are zeros to the
attention, and the error is latched, whatever the number."""

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv4_util import Batch4
from kv_util import BF, HF, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("number", [-1, -2 ** 31, -2 ** 31 + 1, 2 ** 31 - 1])
@pytest.mark.parametrize("four,dtype", [(True, BF), (True, HF), (False, BF), (False, HF)])
@pytest.mark.parametrize("new", [[1, 1], [40, 3]])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_any_bad_number_is_latched(number, four, dtype, new, page):
    lens = [1500, 600]
    b = (Batch4 if four else Batch)(new, lens, 8, 2, 128, page, dtype).fill()
    for r, i in ((0, 0), (0, 600 // page), (1, 200 // page)):  # (none of a new token)
        b.pages[r, i] = number
        lo, hi = i * page, min((i + 1) * page, lens[r])
        b.keys[r][lo:hi] = 0
        b.values[r][lo:hi] = 0
    kv = b.handle()
    kv.check()
    caches = b.caches if four else (b.k_cache, b.v_cache)
    out, lse = kv.paged_attention(b.q, *caches, want_lse=True)
    assert kv.status() == pkg.SMETRIC_ERR_INVALID_ARG and kv.status() == pkg.SMETRIC_OK
    b.assert_attends(out, lse)
    kv.close()
