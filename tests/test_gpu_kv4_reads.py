"""Reading the 4-bit paged cache back: arrays that are dropped while another stream
still reads them, and offsets that no row leads to."""

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv4_util import DEV, Batch4

pytestmark = pytest.mark.gpu
SLEEP = 200_000_000  # cycles: about 0.1 s, longer than the host takes to go on


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("raw", [False, True])
def test_index_arrays_outlive_a_read_on_another_stream(raw):
    """Their memory is not handed out again on the current stream before the read that waits on the other has read them."""
    b = Batch4([1, 1], [300, 70], 8, 2, 64, 16).fill()
    kv = b.handle()
    rows = torch.tensor([0, 200, 250], device=DEV)
    first = torch.tensor([90, 10], dtype=torch.int32, device=DEV)
    want = kv.read(*b.caches, rows, b.pages, 250, first=first)
    kv.check()
    s = torch.cuda.Stream()
    arrays = [x.contiguous().clone() for x in (rows, b.pages, first)]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(s):
        torch.cuda._sleep(SLEEP)
    got = kv.read(*b.caches, arrays[0], arrays[1], 250, first=arrays[2], stream=s.cuda_stream if raw else s)
    like = [(x.shape, x.dtype) for x in arrays]
    del arrays
    others = [torch.zeros(shape, dtype=dtype, device=DEV) for _ in range(4) for shape, dtype in like]  # (positions, pages that there are)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and all(bool((x == 0).all()) for x in others)
    kv.check()
    kv.close()


@pytest.mark.parametrize("offsets", [[0, 40, 80, 121], [0, 120, 120, 500], [0, 120, -1, 120], [0, 120, 130, 120], [120, 120, 120, 1 << 40]])
@pytest.mark.parametrize("wide", [False, True])
def test_bad_offsets_of_requests_without_rows_are_latched(offsets, wide):
    """Also where every row belongs to a request whose own offsets are good; and among many requests."""
    b = Batch4([1, 1, 1], [40, 40, 40], 2, 2, 64, 16).fill()
    kv = b.handle()
    pages = b.pages.clamp(min=0)
    n = 3
    if wide:
        offsets = offsets[:1] + [offsets[0]] * 3000 + offsets[1:]
        pages = pages[:1].repeat(3003, 1)
        n = 3003
    kv.read(*b.caches, torch.tensor(offsets, device=DEV), pages, 120)
    assert len(offsets) == n + 1 and kv.status() == pkg.SMETRIC_ERR_INVALID_ARG and kv.status() == pkg.SMETRIC_OK
    kv.close()


def test_good_offsets_latch_nothing():
    b = Batch4([1, 1, 1], [40, 40, 40], 2, 2, 64, 16).fill()
    kv = b.handle()
    for offsets in ([0, 40, 80, 120], [0, 0, 0, 0], [120, 120, 120, 120], [5, 5, 40, 41], [0, 0, 40, 40]):
        kv.read(*b.caches, torch.tensor(offsets, device=DEV), b.pages, 120)
        kv.check()
    kv.close()
