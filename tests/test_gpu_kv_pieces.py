"""Sequences in many pieces: one unit that all SMs share, of few rows and of
many, and the same bits call after call and plan after plan."""

import pytest
import torch

from kv_util import BF, HF, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("hq,hk,d,new,lens", [
    (32, 4, 128, [1], [24577]), (33, 3, 64, [2, 0, 1], [9000, 7, 15000]), (16, 16, 64, [1] * 32, [800] * 32), (32, 1, 128, [1], [40000]),
    (5, 1, 128, [24], [57191]), (8, 1, 96, [40], [30000]), (4, 4, 32, [31], [6000]), (7, 1, 16, [6], [30000]), (1, 1, 48, [250], [20000]),
])
def test_shared_sequences(hq, hk, d, new, lens):
    for dtype in (BF, HF):
        b = Batch(new, lens, hq, hk, d, 64, dtype, seed=len(lens)).fill()
        kv = b.handle(max_requests=40, max_tokens=300)
        first = None
        for _ in range(3):
            out, lse = kv.paged_attention(b.q, b.k_cache, b.v_cache, want_lse=True)
            kv.check()
            if first is None:
                b.assert_attends(out, lse)
                first = out, lse
            assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
            kv.plan(b.offsets, b.kv_lens, b.pages, b.t)
        kv.close()
