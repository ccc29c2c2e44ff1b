"""Reading the 4-bit paged cache back: arrays that are dropped while another stream
still reads them."""

import pytest
import torch

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
