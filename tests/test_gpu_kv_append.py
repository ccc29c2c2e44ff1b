"""Plan, append and the norm + rotation pass of the paged KV$ operators
against a plain form in 64 bits, slot by slot; what they do not own stays as
it was."""

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv_util import BF, DEV, HF, Batch, assert_close, table, transform64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def _same(a, b):
    """Equal bit for bit (NaN included)."""
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


def _run_append(b, rot, interleaved, q_norm, k_norm, with_q, in_place=False, eps=1e-6):
    g = torch.Generator(device=DEV)
    g.manual_seed(99)
    qkv = (3 * torch.randn(b.t, (b.hq + 2 * b.hk) * b.d, generator=g, device=DEV)).to(b.dtype)
    q, k, v = (x.unflatten(1, (-1, b.d)) for x in qkv.split([b.hq * b.d, b.hk * b.d, b.hk * b.d], 1))
    cs = table(max(b.lens + [1]), rot) if rot else None
    wq, wk = ((1 + 0.3 * torch.randn(b.d, generator=g, device=DEV)).to(b.dtype) for _ in range(2))
    wq, wk = wq if q_norm else None, wk if k_norm else None
    before_k, before_v, before_q = b.k_cache.clone(), b.v_cache.clone(), q.clone()
    kv = b.handle()
    q_out = (q if in_place else torch.full((b.t, b.hq, b.d), 5.0, dtype=b.dtype, device=DEV)) if with_q else None
    kv.append(b.k_cache, b.v_cache, k, v, q=q if with_q else None, q_out=q_out, cos_sin=cs, interleaved=interleaved,
              q_norm=wq, k_norm=wk, eps=eps)
    kv.check()
    want_k, want_v = before_k.clone(), before_v.clone()
    owned = torch.zeros(b.pool, b.page, dtype=torch.bool, device=DEV)
    a = b.first
    for r in range(b.n):
        e, lo = a + b.new[r], b.lens[r] - b.new[r]
        pg, sl = b.slots(r, lo)
        pos = torch.arange(lo, b.lens[r], device=DEV)
        owned[pg, sl] = True
        y, mag = transform64(k[a:e], wk, pos, cs, interleaved, eps)
        assert_close(b.k_cache[pg, sl], y, mag, b.dtype, f"keys of request {r}")
        assert _same(b.v_cache[pg, sl], v[a:e])
        if with_q:
            y, mag = transform64(before_q[a:e], wq, pos, cs, interleaved, eps)
            assert_close(q_out[a:e], y, mag, b.dtype, f"queries of request {r}")
        a = e
    assert _same(b.k_cache[~owned], want_k[~owned]) and _same(b.v_cache[~owned], want_v[~owned])
    if with_q and not in_place:  # tokens of no request
        assert (q_out[:b.first] == 5).all() and (q_out[a:] == 5).all()
    kv.close()


MIX = ([1, 0, 7, 33, 1, 64, 0, 130], [1, 0, 40, 33, 65, 64, 17, 300])


@pytest.mark.parametrize("hq,hk,d", [(4, 4, 128), (32, 4, 128), (7, 1, 64), (10, 2, 96), (3, 3, 16), (6, 2, 48), (64, 8, 80)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_append_head_layouts(hq, hk, d, dtype):
    for k, (rot, il) in enumerate([(d, False), (d, True), (16, False), (0, False)]):
        b = Batch(*MIX, hq, hk, d, 16, dtype, seed=k)
        _run_append(b, rot, il, k % 2 == 0, k < 2, k != 2, in_place=k == 1)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["nhd", "hnd", "pair"])
def test_append_pages_and_strides(page, layout):
    _run_append(Batch(*MIX, 8, 2, 64, page, layout=layout, gap=(3, 5)), 64, False, True, True, True)


def test_append_only_some_norms_and_one_token():
    for qn, kn in [(True, False), (False, True)]:
        _run_append(Batch(*MIX, 4, 2, 96, 32), 32, False, qn, kn, True)
    _run_append(Batch([1], [1], 8, 1, 128, 16), 128, False, True, True, True)
    _run_append(Batch([0, 0], [5, 0], 8, 1, 128, 16), 128, False, True, True, True)


def test_append_many_requests_and_one_long():
    rng = torch.Generator().manual_seed(3)
    new = torch.randint(0, 5, (3000,), generator=rng).tolist()
    lens = [x + int(y) for x, y in zip(new, torch.randint(0, 60, (3000,), generator=rng))]
    _run_append(Batch(new, lens, 4, 2, 64, 16), 64, False, False, True, True)
    _run_append(Batch([20011], [20030], 4, 1, 64, 64), 64, True, True, True, True)


def test_zero_rows_and_large_values():
    """A head of zeros norms to zeros (eps keeps the root from zero); large ones stay finite."""
    kv = pkg.SMetricKV(64, 2, 1, 16, 1, 1, 4, dtype=BF)
    q = torch.zeros(4, 2, 64, dtype=BF, device=DEV)
    q[1] = 1e18
    w = torch.ones(64, dtype=BF, device=DEV)
    out, none = kv.qk_norm_rope(q, None, torch.zeros(4, dtype=torch.int32, device=DEV), q_norm=w)
    kv.check()
    assert none is None and (out[0] == 0).all() and (out[2:] == 0).all()
    assert ((out[1].float() - 1).abs() <= 2.0 ** -8).all()
    kv.close()


@pytest.mark.parametrize("tokens", [0, 1, 2, 31, 1000, 9973])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_norm_rope_alone(tokens, dtype):
    hq, hk, d, rot, eps = 8, 2, 128, 64, 1e-5
    g = torch.Generator(device=DEV)
    g.manual_seed(tokens)
    q, k = (torch.randn(tokens, h + 1, d + 8, generator=g, device=DEV).to(dtype)[:, 1:, 8:] for h in (hq, hk))
    pos = torch.randint(0, 500, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    wq, wk = ((1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(dtype) for _ in range(2))
    cs = table(500, rot)
    kv = pkg.SMetricKV(d, hq, hk, 16, 1, 1, 1, dtype=dtype)
    for il in (False, True):
        qo, ko = kv.qk_norm_rope(q, k, pos, cos_sin=cs, interleaved=il, q_norm=wq, k_norm=wk, eps=eps)
        kv.check()
        for got, x, w in ((qo, q, wq), (ko, k, wk)):
            y, mag = transform64(x, w, pos, cs, il, eps)
            assert_close(got, y, mag, dtype)
    qo, ko = kv.qk_norm_rope(None, k, pos)  # neither: a copy
    assert qo is None and _same(ko, k)
    kv.close()


def test_device_refusals_leave_tokens_out():
    b = Batch([4, 4, 4], [4, 20, 40], 2, 1, 64, 16, junk=9.0)
    k = torch.ones(b.t, 1, 64, dtype=BF, device=DEV)
    kv = b.handle()
    # positions past the table: request 1 is at 16..19, request 2 at 36..39
    kv.append(b.k_cache, b.v_cache, k, k, cos_sin=table(18, 64))
    assert kv.status() == pkg.SMETRIC_ERR_OVERFLOW and kv.status() == pkg.SMETRIC_OK
    assert int((b.v_cache != 9).any(-1).sum()) == 4 + 2
    # a page outside the cache
    for bad in (b.pool, -1):
        b.v_cache.fill_(9.0)
        pages = b.pages.clone()
        pages[1, 1] = bad
        kv.plan(b.offsets, b.kv_lens, pages, b.t)
        assert kv.status() == pkg.SMETRIC_ERR_INVALID_ARG
        kv.append(b.k_cache, b.v_cache, k, k)
        assert kv.status() == pkg.SMETRIC_OK and int((b.v_cache != 9).any(-1).sum()) == 8
    # lengths and offsets that cannot be: nothing is appended
    for off, lens in [([0, 4, 8, 13], [4, 20, 40]), ([0, 4, 8, 12], [3, 20, 40]), ([0, 8, 4, 12], [8, 20, 40]),
                      ([-1, 4, 8, 12], [9, 20, 40]), ([0, 4, 8, 12], [4, 20, 4000]), ([0, 4, 8, 12], [4, -2, 40])]:
        b.v_cache.fill_(9.0)
        kv.plan(torch.tensor(off, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), b.pages, b.t)
        kv.append(b.k_cache, b.v_cache, k, k)
        assert kv.status() == pkg.SMETRIC_ERR_INVALID_ARG
        assert bool((b.v_cache == 9).all())
        out, lse = kv.paged_attention(b.q, b.k_cache, b.v_cache, want_lse=True)
        assert kv.status() == pkg.SMETRIC_OK and bool((out == 0).all()) and bool((lse == -float("inf")).all())
    pos = torch.tensor([0, -1, 18, 17], dtype=torch.int32, device=DEV)
    out = torch.full((4, 1, 64), 9.0, dtype=BF, device=DEV)
    kv.qk_norm_rope(None, k[:4], pos, cos_sin=table(18, 64), k_out=out)
    assert kv.status() == pkg.SMETRIC_ERR_OVERFLOW
    assert (out == 9).all(-1)[:, 0].tolist() == [False, True, True, False]
    kv.close()


def test_host_refusals():
    b = Batch([4], [20], 4, 2, 64, 16)
    kv = pkg.SMetricKV(64, 4, 2, 16, b.pool, 1, 4, dtype=BF)
    k = torch.zeros(4, 2, 64, dtype=BF, device=DEV)
    with pytest.raises(pkg.SmetricError):
        kv.append(b.k_cache, b.v_cache, k, k)  # no plan
    with pytest.raises(pkg.SmetricError):
        kv.paged_attention(b.q, b.k_cache, b.v_cache)
    for off, lens, n_tokens in [(torch.tensor([0, 2, 4], device=DEV), b.kv_lens.repeat(2), 4), (b.offsets, b.kv_lens, 5),
                                (b.offsets, b.kv_lens, -1)]:
        with pytest.raises(pkg.SmetricError):
            kv.plan(off, lens, b.pages.repeat(lens.numel(), 1), n_tokens)
    with pytest.raises(pkg.SmetricError):
        kv.plan(b.offsets, b.kv_lens, b.pages, 4, window=-1)
    kv.plan(b.offsets, b.kv_lens, b.pages, 4)
    wide = torch.zeros(4, 2, 68, dtype=BF, device=DEV)
    for bad in (wide[..., 4:], torch.zeros(4, 2 * 68, dtype=BF, device=DEV).as_strided((4, 2, 64), (136, 68, 1))):
        with pytest.raises(pkg.SmetricError):
            kv.append(b.k_cache, b.v_cache, bad, k)
        with pytest.raises(pkg.SmetricError):
            kv.paged_attention(torch.zeros(4, 4, 68, dtype=BF, device=DEV)[..., 4:], b.k_cache, b.v_cache)
    for bad in (k.half(), k[:3], torch.zeros(4, 2, 32, dtype=BF, device=DEV), torch.zeros(4, 2, 64, 2, dtype=BF, device=DEV)[..., 0]):
        with pytest.raises(ValueError):
            kv.append(b.k_cache, b.v_cache, bad, k)
    with pytest.raises(ValueError):
        kv.append(b.k_cache[:-1], b.v_cache[:-1], k, k)
    for kw in (dict(cos_sin=table(30, 24)), dict(cos_sin=table(30, 80)), dict(k_norm=k[0, 0], eps=float("nan")),
               dict(k_norm=k[0, 0], eps=-1.0)):
        with pytest.raises(pkg.SmetricError):
            kv.append(b.k_cache, b.v_cache, k, k, **kw)
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(pkg.SmetricError):
            kv.paged_attention(b.q, b.k_cache, b.v_cache, scale=scale)
    kv.check()
    before = pkg.smetric_kv_launch_count(kv.handle)
    kv.append(b.k_cache, b.v_cache, k, k)
    assert pkg.smetric_kv_launch_count(kv.handle) == before + 1
    kv.close()


def test_another_stream():
    """Calls go to the stream they are given."""
    b = Batch([5, 300], [70, 900], 8, 2, 64, 16).fill()
    kv = b.handle()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    kv.plan(b.offsets, b.kv_lens, b.pages, b.t, stream=s)
    k, v = torch.cat([x[-n:] for x, n in zip(b.keys, b.new)]), torch.cat([x[-n:] for x, n in zip(b.values, b.new)])
    kv.append(b.k_cache, b.v_cache, k, v, stream=s)
    with torch.cuda.stream(s):
        out = kv.paged_attention(b.q, b.k_cache, b.v_cache)
    kv.check(s)
    b.assert_attends(out)
    kv.close()
