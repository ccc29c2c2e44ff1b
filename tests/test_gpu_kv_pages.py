"""Every page of a long sequence counts: queries that each single out one key,
whose value then is the output, over requests that share the sequence's pages;
and long sequences in half precision, whose finer rounding leaves a wrong page
less room than bf16's."""

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv_util import BF, DEV, HF, TINY, UNIT, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("d,dtype", [(64, BF), (128, HF), (128, BF)])
@pytest.mark.parametrize("requests", [1, 120])
def test_each_page_is_read_in_its_place(page, d, dtype, requests):
    """Keys of one length: a query along a key scores it 4 sqrt(d), 32 or more,
    and the others 4 z, z about normal: they share a weight of 1e-6 or so, and a
    value from another place is off by its own size."""
    length, group = 16001, 8
    g = torch.Generator(device=DEV)
    g.manual_seed(page + d)
    used = -(-length // page)
    pool = used + 3
    order = torch.randperm(pool, generator=g, device=DEV)[:used]
    k, v = (torch.randn(length, d, generator=g, device=DEV) for _ in range(2))
    k = (k * (d ** 0.5 / k.norm(dim=1, keepdim=True))).to(dtype)
    v = v.to(dtype)
    k_cache, v_cache = (torch.full((pool, page, 1, d), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    at = torch.arange(length, device=DEV)
    k_cache[order[at // page], at % page, 0], v_cache[order[at // page], at % page, 0] = k, v
    pages = order.to(torch.int32).repeat(requests, 1)
    kv = pkg.SMetricKV(d, group, 1, page, pool, requests, requests, dtype=dtype)
    kv.plan(torch.arange(requests + 1, device=DEV), torch.full((requests,), length, dtype=torch.int32, device=DEV), pages, requests)
    # a key of each page (or of a sample of pages, the first and the last among them), at a place that moves
    calls = 6 if requests == 1 else 1
    targets = torch.linspace(0, used - 1, calls * requests * group, device=DEV).round().long()
    targets = (targets * page + targets * 7 % page).clamp(max=length - 1).view(calls, requests, group)
    for target in targets:
        q = (4 * k[target].float()).to(dtype)
        out = kv.paged_attention(q, k_cache, v_cache)
        kv.check()
        x = q.double().flatten(0, 1) @ k.double().T * d ** -0.5
        p = x.softmax(-1)
        want, mag = p @ v.double(), p @ v.double().abs()
        # the weights rounded once, the output once; 32-bit scores of up to 45 are (d + 2) 2^-24 45 = 2^-11.5 off at
        # most, which moves a weight and the sum by as much
        u = UNIT[dtype]
        tol = u * want.abs() + (u + 2.0 ** -10) * mag + TINY[dtype]
        off = (out.double().flatten(0, 1) - want).abs() - tol
        assert out.isfinite().all() and (off <= 0).all(), f"{int((off > 0).sum())} values off, by {off.max():.3g}"
        assert (p.gather(1, target.flatten()[:, None]) > 0.99).all()
    kv.close()


@pytest.mark.parametrize("lens", [[30001], [12000, 30, 7000], [5] * 70, [2000] * 11])
@pytest.mark.parametrize("hq,hk,d", [(32, 4, 128), (16, 16, 64)])
def test_long_single_tokens_in_half_precision(lens, hq, hk, d):
    b = Batch([1] * len(lens), lens, hq, hk, d, 32, HF, seed=len(lens)).fill()
    kv = b.handle()
    out, lse = kv.paged_attention(b.q, b.k_cache, b.v_cache, want_lse=True)
    kv.check()
    b.assert_attends(out, lse)
    kv.close()
