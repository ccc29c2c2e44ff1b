"""Attention whose scores are so large that 32 bits round them by a weight's range or
more: a key ahead of the others has the output for itself, up to the largest scores
that the operators take; past them the error is latched."""

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv4_util import DEV, SCALES, Batch4, values64
from kv_util import BF, HF, TINY, UNIT, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


SHAPES = [([1, 1, 1], [3000, 70, 33], 16, 2, 128), ([1, 1], [20011, 45], 12, 1, 64), ([40, 130, 2], [300, 3001, 45], 16, 2, 128), ([300], [5000], 4, 1, 64)]


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("new,lens,hq,hk,d", SHAPES)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("power", [16, 18, 20, 22, 26, 29, 33, 60, 100])
def test_large_scores(four, new, lens, hq, hk, d, dtype, power):
    """Keys of one direction, whose lengths are a 17th or more apart or alike: a row's scores are a number times the
    lengths, alike to the last bit where these are, and else 2^8 or more apart."""
    b = (Batch4 if four else Batch)(new, lens, hq, hk, d, 16, dtype)
    g = torch.Generator(device=DEV)
    g.manual_seed(power)
    sign = torch.randint(0, 2, (hk, d), generator=g, device=DEV)  # e2m1: 2 is 1, 10 is -1
    lengths = SCALES.to(DEV)[40:72]
    for r, n in enumerate(lens):
        pick = torch.randint(0, 32, (n, hk), generator=g, device=DEV)
        if four:
            bits = (40 + pick)[..., None].expand(n, hk, d // 16)
            b.held[0][r] = (2 + 8 * sign).expand(n, hk, d), bits
            b.keys[r] = values64(*b.held[0][r])
        else:
            b.keys[r] = ((1 - 2 * sign).double() * lengths[pick][..., None]).to(dtype)
    b.fill()
    # (a row's product with the direction: a whole number that is not 0)
    q = torch.randint(-3, 4, b.q.shape, generator=g, device=DEV).to(dtype)
    along = (q.double().view(b.t, hk, -1, d) * (1 - 2 * sign).double()[:, None]).sum(-1).view(b.t, hq)
    q[..., 0] += torch.where(along == 0, 1, 0).to(dtype)
    b.q = q
    scale = 2.0 ** power
    kv = b.handle()
    out, lse = kv.paged_attention(b.q, *((b.caches if four else (b.k_cache, b.v_cache))), scale=scale, want_lse=True)
    status = kv.status()
    kv.close()
    want, want_lse, mag = b.attend64(scale)
    # half precision's weights, which caches in 4 bits have for either type, take 2^27, those in bf16 2^29
    limit = 2.0 ** 27 if four or dtype == HF else 2.0 ** 29
    largest = float(want_lse[want_lse.isfinite()].abs().max())
    if largest >= limit and status != pkg.SMETRIC_OK or largest >= 2 * limit:
        assert status == pkg.SMETRIC_ERR_OVERFLOW
        return
    assert status == pkg.SMETRIC_OK
    assert bool(out.isfinite().all()) and bool(lse.isfinite().all())
    u = UNIT[dtype]  # (weights of keys alike are equal: their rounding is one factor of all; as the other attention tests have it)
    off = (out.double() - want).abs() - (u * want.abs() + (u + 2.0 ** -12) * mag + TINY[dtype])
    assert bool((off <= 0).all()), f"{int((off > 0).sum())} of {off.numel()} values off, by {off.max():.3g}"
    # a score is a sum of whole numbers times a length, which is exact; the factor with log2 e, the product, the
    # logarithm and the factor ln 2 are rounded, 2^-24 of the score each, and once more by their sum
    err = (lse.double() - want_lse).abs() - (2.0 ** -21 * want_lse.abs() + 2.0 ** -12)
    assert bool((err <= 0).all()), f"lse off by {err.max():.3g}"
