"""Query rows at the ends of their range over the 4-bit paged cache: zeros and the
smallest numbers, with scales and exponents that leave next to nothing of a score; and
small elements beside a large one."""

import pytest
import torch

from kv4_util import DEV, Batch4, values64
from kv_util import BF, HF

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def with_exp(b, exp):
    """The batch with its keys' codes and scales under another exponent."""
    b.caches[0] = b.caches[0]._replace(exp=exp)
    b.keys = [values64(*h, exp) for h in b.held[0]]
    return b


def check(b, scale=None):
    kv = b.handle()
    out, lse = kv.paged_attention(b.q, *b.caches, scale=scale, want_lse=True)
    kv.check()
    b.assert_attends(out, lse, scale)
    kv.close()


# (all off a tile, so that the last one has keys that are not seen)
SHAPES = [([1, 1, 1, 1], [3000, 70, 33, 1], 16, 2, 128), ([1, 1], [500, 45], 12, 1, 64), ([2, 1], [90, 20], 4, 1, 32), ([40, 130], [300, 401], 16, 2, 128),
          ([20, 3], [77, 60], 40, 1, 64)]


@pytest.mark.parametrize("new,lens,hq,hk,d", SHAPES)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("exp,scale", [(0, None), (0, 1e-8), (0, 1e-30), (0, 2.0 ** -149), (-21, None), (-22, None), (-64, None), (-64, 2.0 ** -60),
                                       (64, None), (64, 2.0 ** 60)])
def test_rows_of_zeros_and_of_the_smallest_numbers(new, lens, hq, hk, d, dtype, exp, scale):
    """Rows of zeros see the mean of the values; so do others whose scores are next to nothing."""
    b = with_exp(Batch4(new, lens, hq, hk, d, 16, dtype).fill(), exp)
    factor = (d ** -0.5 if scale is None else scale) * 2.0 ** exp
    sizes = [0.0] + [s for s in ([2.0 ** -133, 2.0 ** -126, 2.0 ** -100, 2.0 ** -64, 2.0 ** -20, 1.0, 2.0 ** 60] if dtype == BF else
                                 [2.0 ** -24, 2.0 ** -14, 2.0 ** -7, 1.0]) if s * factor <= 1.0]
    pick = torch.arange(b.t * hq, device=DEV).view(b.t, hq) * 7 % (3 * len(sizes)) % len(sizes)
    b.q = (b.q.double() * torch.tensor(sizes, dtype=torch.float64, device=DEV)[pick][..., None]).to(dtype)
    assert bool((b.q == 0).all(-1).any()) and bool(b.q.isfinite().all())
    check(b, scale)


@pytest.mark.parametrize("new,lens,hq,hk,d", SHAPES)
@pytest.mark.parametrize("lift", [12, 24])
def test_small_elements_beside_a_large_one(new, lens, hq, hk, d, lift):
    """Half-precision queries whose largest element meets zeros alone: the others make the scores, with all their bits."""
    b = Batch4(new, lens, hq, hk, d, 16, HF)
    for r in range(b.n):
        b.held[0][r][0][..., 5] = 0
        b.keys[r] = values64(*b.held[0][r])
    b.fill()
    b.q = (b.q.double() * 2.0 ** -lift * 2.0 ** 8).to(HF)
    b.q[..., 5] = 2.0 ** 15
    check(b, d ** -0.5 * 2.0 ** (lift - 8))
