"""Which kernel takes a request of a batch over the 4-bit paged cache: its own new
tokens decide, not the batch's."""

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


@pytest.mark.parametrize("hq,hk,d,dtype", [(16, 2, 128, BF), (16, 1, 64, HF), (4, 4, 32, BF), (10, 2, 96, HF)])
@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("slots,singles", [(200, 0), (260, 0), (260, 30), (230, 30)])
def test_empty_requests_leave_a_chunk_as_it_is(hq, hk, d, dtype, window, slots, singles):
    """A chunk's output is the same, bit for bit, alone and among as many requests as there are tokens or more, whether
    these have a token each or none. (Rows that go through the two kernels' sums differ in some last bit.)"""
    new, length = 200, 700
    alone = Batch4([new], [length], hq, hk, d, 16, dtype, window=window)
    b = Batch4([1] * singles + [new] + [0] * (slots - singles - 1), [40] * singles + [length] + [17] * (slots - singles - 1), hq, hk, d, 16, dtype,
               window=window)
    b.q[singles:singles + new] = alone.q
    for i in range(2):
        b.held[i][singles] = alone.held[i][0]
    b.keys[singles], b.values[singles] = alone.keys[0], alone.values[0]
    assert b.t <= b.n
    got = []
    for x in (alone.fill(), b.fill()):
        kv = x.handle()
        out, lse = kv.paged_attention(x.q, *x.caches, want_lse=True)
        kv.check()
        x.assert_attends(out, lse)
        kv.close()
        got.append((out, lse))
    (out, lse), (among, lse_among) = got
    assert torch.equal(among[singles:singles + new], out) and torch.equal(lse_among[singles:singles + new], lse)


@pytest.mark.parametrize("hq,hk,d", [(16, 2, 128), (16, 1, 64), (4, 4, 32), (40, 1, 64)])
def test_single_tokens_that_are_said_to_be(hq, hk, d):
    """The same outputs, bit for bit, by fewer launches where a kernel for few rows takes them all."""
    b = Batch4([1] * 40 + [0] * 10, [30 * i + 1 for i in range(50)], hq, hk, d, 16, gap=(3, 2)).fill()
    kv = b.handle()
    got, launches = [], []
    for max_new in (None, 1, 100):
        kv.plan(b.offsets, b.kv_lens, b.pages, b.t, max_new=max_new)
        before = pkg.smetric_kv_launch_count(kv.handle)
        got.append(kv.paged_attention(b.q, *b.caches, want_lse=True))
        launches.append(pkg.smetric_kv_launch_count(kv.handle) - before)
        kv.check()
    b.assert_attends(*got[0])
    assert all(torch.equal(x, y) for g in got[1:] for x, y in zip(g, got[0]))
    assert launches == ([3, 2, 3] if hq // hk <= 16 else [2, 2, 2])
    kv.close()


@pytest.mark.parametrize("four", [True, False])
def test_more_new_tokens_than_were_said(four):
    """An error of the batch, as bad offsets are; the most that was said is none."""
    b = (Batch4 if four else Batch)([1, 5, 0], [40, 70, 30], 8, 2, 64, 16).fill()
    kv = b.handle()
    caches = b.caches if four else (b.k_cache, b.v_cache)
    for max_new, good in ((5, True), (4, False), (1, False), (0, False), (2 ** 70, True)):
        kv.plan(b.offsets, b.kv_lens, b.pages, b.t, max_new=max_new)
        out, lse = kv.paged_attention(b.q, *caches, want_lse=True)
        assert kv.status() == (pkg.SMETRIC_OK if good else pkg.SMETRIC_ERR_INVALID_ARG)
        if good:
            b.assert_attends(out, lse)
        else:
            assert bool((out == 0).all()) and bool(lse.isinf().all())
    with pytest.raises(pkg.SmetricError):
        kv.plan(b.offsets, b.kv_lens, b.pages, b.t, max_new=-1)
    kv.close()
