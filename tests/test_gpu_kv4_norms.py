"""Queries on their way past the 4-bit paged cache: the append hands on what the
transform alone and the append to 16-bit caches give."""

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv4_util import DEV, Batch4
from kv_util import BF, HF, table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("interleaved", [False, True])
def test_queries_are_those_of_the_transform_alone(d, dtype, interleaved):
    b = Batch4([700, 1, 300], [900, 40, 300], 32, 4, d, 32, dtype, seed=d)
    kv = b.handle()
    wide = pkg.SMetricKV(d, 32, 4, 32, b.pool, b.n, b.t, dtype=dtype)
    wide.plan(b.offsets, b.kv_lens, b.pages, b.t)
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    k, v = (torch.randn(b.t, 4, d, generator=g, device=DEV).to(dtype) for _ in range(2))
    weights = [(1 + torch.randn(d, generator=g, device=DEV) / 8).to(dtype) for _ in range(2)]
    kw = dict(cos_sin=table(1000, d), q_norm=weights[0], k_norm=weights[1], interleaved=interleaved)
    pos = torch.cat([torch.arange(n - m, n, device=DEV) for m, n in zip(b.new, b.lens)]).to(torch.int32)
    q = kv.append(*b.caches, k, v, q=b.q, **kw)
    alone, _ = kv.qk_norm_rope(b.q, k, pos, **kw)
    cache = torch.zeros(2, b.pool, 32, 4, d, dtype=dtype, device=DEV)
    other = wide.append(*cache, k, v, q=b.q, **kw)
    kv.check(), wide.check()
    assert torch.equal(q, alone) and torch.equal(q, other)
    kv.close(), wide.close()
