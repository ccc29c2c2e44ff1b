"""Attention over the 4-bit paged cache against 64-bit arithmetic on what the
codes and scales stand for."""

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv4_util import DEV, Batch4
from kv_util import BF, HF

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def check(b, scale=None, ctx=""):
    kv = b.handle()
    out, lse = kv.paged_attention(b.q, *b.caches, scale=scale, want_lse=True)
    again = kv.paged_attention(b.q, *b.caches, scale=scale)
    kv.check()
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    b.assert_attends(out, lse, scale, ctx)
    kv.close()


HEADS = [(8, 1, 128), (32, 4, 128), (4, 4, 64), (7, 1, 96), (16, 1, 32), (15, 3, 128), (16, 16, 32), (12, 1, 64), (34, 2, 64),
         (40, 1, 128), (128, 1, 64), (5, 5, 96)]


@pytest.mark.parametrize("hq,hk,d", HEADS)
@pytest.mark.parametrize("dtype", [BF, HF])
def test_single_tokens(hq, hk, d, dtype):
    lens = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 300, 1000]
    check(Batch4([1] * len(lens), lens, hq, hk, d, 16, dtype, exps=(1, -2)).fill())


@pytest.mark.parametrize("hq,hk,d", HEADS)
@pytest.mark.parametrize("dtype", [BF, HF])
def test_chunks(hq, hk, d, dtype):
    new = [2, 3, 5, 17, 64, 130, 0, 1]
    lens = [2, 40, 5, 200, 64, 401, 30, 77]
    check(Batch4(new, lens, hq, hk, d, 16, dtype).fill())


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["nhd", "hnd", "pair"])
def test_pages_and_strides(page, layout):
    new, lens = [1, 0, 7, 33, 1, 64, 0, 130], [1, 0, 40, 33, 65, 64, 17, 300]
    check(Batch4(new, lens, 8, 2, 128, page, layout=layout, gap=(3, 5)).fill())
    check(Batch4([1] * 8, [x + 1 for x in lens], 8, 2, 64, page, layout=layout, gap=(2, 0)).fill())


@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 64, 100, 128, 129])
def test_windows(window):
    new, lens = [1, 1, 1, 40, 130, 3, 0], [1, 64, 500, 300, 130, 90, 9]
    for hq, hk, d in [(8, 1, 128), (4, 4, 64), (32, 2, 64)]:
        check(Batch4(new, lens, hq, hk, d, 16, window=window).fill())
        check(Batch4([1] * 7, [x + 1 for x in lens], hq, hk, d, 32, window=window).fill())


@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_long_single_tokens(d):
    """Sequences that many SMs share."""
    for n, length, hq, hk in [(1, 20011, 8, 1), (2, 30001, 16, 2), (3, 5000, 8, 8), (1, 4099, 64, 4)]:
        check(Batch4([1] * n, [length - 7 * i for i in range(n)], hq, hk, d, 64, seed=n).fill())


def test_long_chunks():
    check(Batch4([300, 1], [4000, 5000], 16, 2, 128, 16).fill())
    check(Batch4([700], [700], 8, 2, 64, 32, HF).fill())


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("peak,scale", [(30.0, None), (0.01, None), (1.0, 3.0), (1.0, 1e-4)])
def test_sharp_and_flat_softmax(dtype, peak, scale):
    """Scores of some hundreds, whose errors are by as much larger; and of next to nothing."""
    d = 64
    b = Batch4([1, 1, 20], [700, 33, 300], 8, 2, d, 16, dtype, peak=peak).fill()
    if peak == 30.0:
        scale = d ** -0.5 / 30
    if scale == 3.0:
        b.q = b.q / 24
    check(b, scale)
