"""Attention over the paged cache against a plain form in 64 bits: head
layouts, lengths from none to long, page and tile boundaries, windows, chunks
and single tokens in one batch, junk where no key lies."""

import random

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv_util import BF, DEV, HF, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def _check(b, **kw):
    kv = b.fill().handle()
    out, lse = kv.paged_attention(b.q, b.k_cache, b.v_cache, want_lse=True, **kw)
    kv.check()
    b.assert_attends(out, lse, scale=kw.get("scale"))
    again = kv.paged_attention(b.q, b.k_cache, b.v_cache, **kw)
    assert torch.equal(out, again)  # the same bits call after call
    kv.check()
    kv.close()
    return out


EDGES = ([1, 1, 1, 1, 1, 1, 1, 1, 0, 1, 0], [1, 2, 15, 16, 17, 127, 128, 129, 0, 1000, 300])
CHUNKS = ([1, 2, 16, 17, 0, 127, 128, 129, 300, 33, 260], [1, 2, 16, 20, 9, 127, 400, 129, 300, 1033, 2048])


@pytest.mark.parametrize("hq,hk,d", [(4, 4, 128), (32, 4, 128), (64, 4, 64), (7, 1, 64), (10, 2, 96), (3, 3, 16), (6, 2, 48),
                                     (40, 8, 80), (128, 1, 32), (33, 1, 112)])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("batch", [EDGES, CHUNKS], ids=["steps", "chunks"])
def test_head_layouts(hq, hk, d, dtype, batch):
    _check(Batch(*batch, hq, hk, d, 16, dtype, seed=hq + d))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["nhd", "hnd", "pair"])
@pytest.mark.parametrize("batch", [EDGES, CHUNKS], ids=["steps", "chunks"])
def test_pages_and_strides(page, layout, batch):
    _check(Batch(*batch, 8, 2, 64, page, layout=layout, gap=(2, 3), seed=page))


@pytest.mark.parametrize("window", [1, 2, 16, 127, 128, 129, 500, 5000])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_windows(window, dtype):
    """Pages before the window hold junk and are named by no entry that is used."""
    for batch in (EDGES, CHUNKS, ([700, 1, 300], [4000, 4100, 300])):
        b = Batch(*batch, 14, 2, 128, 32, dtype, window=window, seed=window).fill()
        for r, (n, kv) in enumerate(zip(b.new, b.lens)):
            unused = max(0, kv - n - window + 1) // b.page if n else 0
            b.pages[r, :unused] = -3
        h = b.handle()
        out, lse = h.paged_attention(b.q, b.k_cache, b.v_cache, want_lse=True)
        h.check()
        b.assert_attends(out, lse)
        h.close()


@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_junk_where_no_key_lies(junk):
    for batch in (EDGES, CHUNKS):
        _check(Batch(*batch, 8, 1, 128, 64, junk=junk, seed=5))


@pytest.mark.parametrize("lens", [[30001], [12000, 30, 7000], [5] * 70, [2000] * 11])
@pytest.mark.parametrize("hq,hk,d", [(32, 4, 128), (16, 16, 64)])
def test_long_single_tokens(lens, hq, hk, d):
    """Sequences that several SMs share, and more requests than they are."""
    _check(Batch([1] * len(lens), lens, hq, hk, d, 32, seed=len(lens)))


@pytest.mark.parametrize("new,lens", [([2048], [9000]), ([1500, 40], [1500, 6000]), ([300] * 6, [4000] * 6), ([17], [20000])])
@pytest.mark.parametrize("hq,hk,d", [(16, 2, 128), (4, 4, 64)])
def test_long_chunks(new, lens, hq, hk, d):
    _check(Batch(new, lens, hq, hk, d, 64, seed=sum(new)))


def test_peaked_and_growing_scores():
    """Softmax statistics that move: the largest score comes late, early, and far above the rest."""
    for peak in (6.0, 20.0):
        for seed in range(3):
            b = Batch([1, 200, 40], [3000, 1500, 900], 8, 2, 64, 16, seed=seed, peak=peak / 4)
            for k in b.keys:
                ramp = torch.linspace(0.1, 2.0, k.shape[0], device=DEV)[:, None, None]
                k.copy_((k.float() * (ramp if seed == 0 else ramp.flip(0) if seed == 1 else 1)).to(k.dtype))
                if seed == 2:
                    k[k.shape[0] // 2] *= 4
            _check(b)


def test_equal_scores_and_scale():
    b = Batch(*CHUNKS, 8, 2, 64, 16)
    b.q.zero_()
    _check(b)
    _check(Batch(*CHUNKS, 8, 2, 64, 16, seed=8), scale=0.5)


def test_random_batches():
    rng = random.Random(11)
    for seed in range(30):
        hk = rng.choice([1, 2, 3, 4, 8])
        n = rng.randint(1, 12)
        top = rng.choice([3, 40, 600])
        new = [rng.choice([0, 1, rng.randint(0, top)]) for _ in range(n)]
        lens = [x + rng.choice([0, rng.randint(0, 40), rng.randint(0, 4000)]) for x in new]
        _check(Batch(new, lens, hk * rng.choice([1, 2, 3, 5, 7, 8, 16]), hk, rng.choice([16, 64, 96, 128]),
                     rng.choice([16, 32, 64, 128, 256]), rng.choice([BF, HF]), rng.choice(["nhd", "hnd", "pair"]), seed=seed,
                     window=rng.choice([0, 0, rng.randint(1, 3000)]), gap=(rng.randint(0, 3), rng.randint(0, 3))))


def test_strided_queries_and_outputs():
    b = Batch(*CHUNKS, 8, 2, 96, 16).fill()
    kv = b.handle()
    wide = torch.zeros(b.t, 12, 104, dtype=BF, device=DEV)
    wide[:, 2:10, 8:] = b.q
    out = torch.full((8, b.t, 112), 7.0, dtype=BF, device=DEV)
    kv.paged_attention(wide[:, 2:10, 8:], b.k_cache, b.v_cache, out=out[..., 16:].transpose(0, 1))
    kv.check()
    b.assert_attends(out[..., 16:].transpose(0, 1))
    assert (out[..., :16] == 7).all()
    kv.close()


def test_offsets_past_32_bits():
    """A cache whose pages lie past 2^31 elements and 2^32 bytes."""
    b = Batch([1, 200], [500, 900], 8, 2, 64, 64, seed=4)
    stride = 2 ** 31 // 16 + 64
    k, v = (torch.zeros(b.pool * stride + 64 * 128, dtype=BF, device=DEV) for _ in range(2))
    assert b.pool > 17
    b.k_cache, b.v_cache = (x.as_strided((b.pool, 64, 2, 64), (stride, 128, 64, 1)) for x in (k, v))
    new_k, new_v = (torch.cat([x[r][-n:] for r, n in enumerate(b.new)]) for x in (b.keys, b.values))
    for r in range(b.n):
        pg, sl = b.slots(r, 0, b.lens[r] - b.new[r])
        b.k_cache[pg, sl] = b.keys[r][:-b.new[r]]
        b.v_cache[pg, sl] = b.values[r][:-b.new[r]]
    kv = b.handle()
    kv.append(b.k_cache, b.v_cache, new_k, new_v)
    out, lse = kv.paged_attention(b.q, b.k_cache, b.v_cache, want_lse=True)
    kv.check()
    b.assert_attends(out, lse)
    kv.close()


def test_pages_outside_the_cache_are_latched():
    b = Batch([1, 140], [300, 300], 8, 2, 64, 16).fill()
    kv = b.handle()
    good = kv.paged_attention(b.q, b.k_cache, b.v_cache)
    kv.check()
    b.pages[0, 3] = b.pool  # (the plan reads the entries of new tokens only)
    out = kv.paged_attention(b.q, b.k_cache, b.v_cache)
    assert kv.status() == pkg.SMETRIC_ERR_INVALID_ARG
    assert torch.equal(out[1:], good[1:])
    kv.close()


def test_two_handles_and_new_plans():
    """A handle's plan is its own, and a new plan replaces it."""
    a, b = Batch(*EDGES, 8, 2, 64, 16, seed=1).fill(), Batch(*CHUNKS, 16, 2, 128, 32, seed=2).fill()
    ka, kb = a.handle(max_tokens=5000, max_requests=50), b.handle()
    for _ in range(2):
        a.assert_attends(ka.paged_attention(a.q, a.k_cache, a.v_cache))
        b.assert_attends(kb.paged_attention(b.q, b.k_cache, b.v_cache))
    ka.check(), kb.check()
    c = Batch([100, 1, 50], [101, 30, 50], 8, 2, 64, 16, seed=3, spare_pages=a.pool - 13).fill()
    assert c.pool == a.pool
    ka.plan(c.offsets, c.kv_lens, c.pages, c.t)
    c.assert_attends(ka.paged_attention(c.q, c.k_cache, c.v_cache))
    ka.check()
    ka.close(), kb.close()


def test_captured_in_a_graph():
    b = Batch([1] * 6 + [90], [50, 600, 1, 129, 4000, 70, 800], 8, 2, 64, 16).fill()
    kv = b.handle()
    kv.paged_attention(b.q, b.k_cache, b.v_cache)
    out = torch.zeros(b.t, 8, 64, dtype=BF, device=DEV)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kv.plan(b.offsets, b.kv_lens, b.pages, b.t)
        kv.paged_attention(b.q, b.k_cache, b.v_cache, out=out)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        b.assert_attends(out)
    kv.check()
    kv.close()
