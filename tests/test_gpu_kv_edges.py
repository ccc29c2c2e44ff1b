"""Edges of the paged KV$ operators: NaN rows, positions and lengths at the ends
of their ranges, tables without rows, views of one token or one head, and calls
on another stream than torch's current one."""

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv_util import BF, DEV, HF, UNIT, Batch, table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("hq,hk,d,new,lens", [
    (8, 2, 64, [1, 1], [100, 3]),             # nobody shares them
    (8, 2, 64, [300], [300]),                 # two tiles of queries
    (64, 64, 128, [1], [24577]),              # some two pieces each (of 152 SMs)
    (32, 16, 64, [1], [24577]),               # nine or ten
    (32, 4, 128, [1], [24577]),               # 38
    (16, 2, 128, [40], [30000]),              # of many rows
])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_a_nan_query_stays_nan(hq, hk, d, new, lens, dtype):
    """However many SMs share its keys; the rows beside it are as without it."""
    b = Batch(new, lens, hq, hk, d, 64, dtype, seed=hk).fill()
    kv = b.handle()
    good, good_lse = kv.paged_attention(b.q, b.k_cache, b.v_cache, want_lse=True)
    kv.check()
    b.assert_attends(good, good_lse)
    for token, head in ((0, 0), (b.t - 1, hq - 1), (b.t // 2, hq // 2)):
        q = b.q.clone()
        q[token, head, d // 2] = float("nan")
        out, lse = kv.paged_attention(q, b.k_cache, b.v_cache, want_lse=True)
        kv.check()
        assert bool(out[token, head].isnan().all()) and bool(lse[token, head].isnan())
        out[token, head], lse[token, head] = good[token, head], good_lse[token, head]
        assert torch.equal(out, good) and torch.equal(lse, good_lse)
    kv.close()


@pytest.mark.parametrize("tokens", [0, 1, 5])
def test_a_table_without_rows_latches_every_token(tokens):
    """Every position is past its end: nothing is left unrotated without a word."""
    b = Batch([tokens], [tokens + 20], 4, 2, 64, 16, junk=9.0)
    kv = b.handle()
    k, empty, late = b.q[:, :2] + 1, table(0, 64), pkg.SMETRIC_ERR_OVERFLOW if tokens else pkg.SMETRIC_OK
    q_out = torch.full_like(b.q, 5.0)
    kv.append(b.k_cache, b.v_cache, k, k, q=b.q, q_out=q_out, cos_sin=empty)
    assert kv.status() == late
    assert bool((b.k_cache == 9).all()) and bool((b.v_cache == 9).all()) and bool((q_out == 5).all())
    kv.qk_norm_rope(b.q, None, torch.arange(tokens, dtype=torch.int32, device=DEV), cos_sin=empty, q_out=q_out)
    assert kv.status() == late and bool((q_out == 5).all())
    kv.append(b.k_cache, b.v_cache, k, k, cos_sin=table(30, 0))  # a rotation of no elements is none
    assert kv.status() == pkg.SMETRIC_OK and int((b.k_cache != 9).any(-1).sum()) == 2 * tokens
    kv.close()


@pytest.mark.parametrize("window", [100, 400])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_the_longest_sequence(window, dtype):
    """A request of 2^31 - 1 tokens, of which a window is seen: NaN in the one
    slot past its end and before the window."""
    d, page, new, kv_len = 16, 256, 3, 2 ** 31 - 1
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dtype)  # noqa: E731
    pages = torch.full((1, 2 ** 31 // page), -7, dtype=torch.int32, device=DEV)
    pages[0, -2:] = torch.tensor([1, 2], dtype=torch.int32)
    k_cache, v_cache = (torch.full((4, page, 1, d), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    last = 2 * page - 1  # places in the two pages that are seen, in a row: the one past the end
    for c in (k_cache, v_cache):
        c[1:3].view(2 * page, 1, d)[last - new - window + 1:last - new] = rnd(window - 1, 1, d)
    k, v, q = rnd(new, 1, d), rnd(new, 1, d), rnd(new, 2, d)
    kv = pkg.SMetricKV(d, 2, 1, page, 4, 1, new, dtype=dtype)
    kv.plan(torch.tensor([0, new], device=DEV), torch.tensor([kv_len], dtype=torch.int32, device=DEV), pages, new, window=window)
    kv.append(k_cache, v_cache, k, v)
    out, lse = kv.paged_attention(q, k_cache, v_cache, want_lse=True)
    kv.check()
    keys, values = (c[1:3].view(2 * page, d) for c in (k_cache, v_cache))
    for x, y in ((keys, k), (values, v)):
        assert torch.equal(x[last - new:last], y[:, 0]) and bool(x[last].isnan().all())
    for i in range(new):
        end = last - new + i + 1  # past its own place
        x = q[i].double() @ keys[end - window:end].double().T * d ** -0.5
        p = x.softmax(-1)
        want, mag = p @ values[end - window:end].double(), p @ values[end - window:end].double().abs()
        u = UNIT[dtype]  # (the bound that the other attention tests use)
        assert bool(((out[i].double() - want).abs() <= u * want.abs() + (u + 2.0 ** -12) * mag).all())
        assert bool(((lse[i].double() - x.logsumexp(-1)).abs() <= 2.0 ** -12).all())
    kv.close()


@pytest.mark.parametrize("cos_sin", [False, True])
def test_negative_positions_are_left_out(cos_sin):
    """With a table and without one."""
    q = torch.randn(4, 2, 64, device=DEV).to(BF)
    w = torch.ones(64, dtype=BF, device=DEV)
    kv = pkg.SMetricKV(64, 2, 2, 16, 1, 1, 1)
    for pos in ([0, -1, 17, 3], [-2 ** 31, 1, 2, 3]):
        at = torch.tensor(pos, dtype=torch.int32, device=DEV)
        q_out, k_out = torch.full_like(q, 9.0), torch.full_like(q, 9.0)
        kv.qk_norm_rope(q, q, at, cos_sin=table(18, 64) if cos_sin else None, q_norm=w, q_out=q_out, k_out=k_out)
        assert kv.status() == pkg.SMETRIC_ERR_OVERFLOW
        left = torch.tensor(pos, device=DEV) < 0
        for out in (q_out, k_out):
            assert torch.equal((out == 9).all(-1).all(-1), left)
    kv.close()


def _views(tokens, heads, d, seed=0):
    """Random [tokens, heads, d] tensors whose dimension of one, if any, comes first, second or last in memory."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    flat = torch.randn(tokens * heads, d, generator=g, device=DEV).to(BF)
    if tokens == 1:
        yield flat.unsqueeze(2).permute(2, 0, 1)  # a token stride of 1
        yield flat.unsqueeze(1).transpose(0, 1)
        yield torch.randn(heads, 9, d, generator=g, device=DEV).to(BF)[:, 4:5].transpose(0, 1)
    if heads == 1:
        yield flat.unsqueeze(2).transpose(1, 2)  # a head stride of 1
        yield flat.unsqueeze(0).transpose(0, 1)
        yield torch.randn(tokens, 3 * d, generator=g, device=DEV).to(BF)[:, d:2 * d].unsqueeze(1)


@pytest.mark.parametrize("tokens,hq", [(1, 1), (1, 4), (7, 1)])
def test_views_of_one_token_or_one_head(tokens, hq):
    """The stride of a dimension of one is arbitrary, and torch gives a new tensor the same one."""
    b = Batch([tokens], [tokens + 300], hq, 1, 64, 16).fill()
    kv = b.handle()
    pos = torch.arange(tokens, dtype=torch.int32, device=DEV)
    kw = dict(cos_sin=table(400, 64), q_norm=torch.ones(64, dtype=BF, device=DEV))
    for q in _views(tokens, hq, 64):
        plain = q.contiguous().view(-1).view(tokens, hq, 64).clone()
        for k in _views(tokens, 1, 64, seed=1) if tokens > 1 else [torch.ones(1, 1, 64, dtype=BF, device=DEV)]:
            got = kv.qk_norm_rope(q, k, pos, **kw)
            want = kv.qk_norm_rope(plain, k.contiguous().view(-1).view(tokens, 1, 64).clone(), pos, **kw)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            caches = [(b.k_cache.clone(), b.v_cache.clone()) for _ in range(2)]
            got = kv.append(*caches[0], k, k, q=q, **kw)
            want = kv.append(*caches[1], k.contiguous().clone(), k.contiguous().clone(), q=plain, **kw)
            assert torch.equal(got, want)
            assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(*caches))
        got, want = (kv.paged_attention(x, b.k_cache, b.v_cache, want_lse=True) for x in (q, plain))
        kv.check()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    kv.close()


SLEEP = 200_000_000  # cycles: about 0.1 s, longer than the host takes to go on


def _calls(kv, b, stream):
    """Every call that allocates, on a stream: its new tensors."""
    pos = torch.arange(b.t, dtype=torch.int32, device=DEV)
    k, v = (torch.cat([x[-n:] for x, n in zip(xs, b.new)]) for xs in (b.keys, b.values))
    torch.cuda.synchronize()
    return [
        lambda: list(kv.paged_attention(b.q, b.k_cache, b.v_cache, want_lse=True, stream=stream)),
        lambda: [kv.append(b.k_cache, b.v_cache, k, v, q=b.q, stream=stream)],
        lambda: list(kv.qk_norm_rope(b.q, k, pos, stream=stream)),
    ]


@pytest.mark.parametrize("raw", [False, True])
def test_new_outputs_on_another_stream(raw):
    """Their memory is not handed out again before that stream has written it,
    nor written before the current stream is done with its last owner."""
    b = Batch([40, 1], [300, 70], 8, 2, 64, 16).fill()
    s = torch.cuda.Stream()
    kv = b.handle()
    for call in _calls(kv, b, s.cuda_stream if raw else s):
        got = call()
        torch.cuda.synchronize()
        like = [x.clone() for x in got]
        del got
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        # dropped before they are written
        with torch.cuda.stream(s):
            torch.cuda._sleep(SLEEP)
        call()
        others = [torch.full_like(x, 7.0) for x in like for _ in range(2)]
        torch.cuda.synchronize()
        assert all(bool((x == 7).all()) for x in others)
        del others
        torch.cuda.empty_cache()
        # memory whose last owner is still being read
        owners = [torch.full_like(x, 3.0) for x in like for _ in range(2)]
        copies = [torch.empty_like(x) for x in owners]
        torch.cuda.synchronize()
        torch.cuda._sleep(SLEEP)
        for c, x in zip(copies, owners):
            c.copy_(x)
        del owners, x
        got = call()
        torch.cuda.synchronize()
        assert all(bool((c == 3).all()) for c in copies)
        assert all(torch.equal(x, y) for x, y in zip(got, like))
        del got, copies, like
    kv.check()
    kv.close()


def test_new_outputs_used_on_the_current_stream():
    """Read there while the stream that wrote them allocates again."""
    b = Batch([40, 1], [300, 70], 8, 2, 64, 16).fill()
    s = torch.cuda.Stream()
    kv = b.handle()
    for call in _calls(kv, b, s):
        got = call()
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        want = [x.clone() for x in got]
        copies = [torch.empty_like(x) for x in got]
        torch.cuda.synchronize()
        torch.cuda._sleep(SLEEP)
        for c, x in zip(copies, got):
            c.copy_(x)
        del got, x
        with torch.cuda.stream(s):
            others = [torch.full_like(x, 7.0) for x in want for _ in range(2)]
        torch.cuda.synchronize()
        assert all(torch.equal(c, w) for c, w in zip(copies, want))
        del others, want, copies
    kv.check()
    kv.close()


@pytest.mark.parametrize("how", ["stream", "raw", "current"])
def test_a_plans_tensors_outlive_the_attention_on_another_stream(how):
    """A new plan drops them: their memory is not handed out again before an
    attention that still waits on that stream has read the page numbers."""
    b = Batch([1, 40, 1], [300, 800, 70], 8, 2, 64, 16).fill()
    kv = b.handle()
    want = kv.paged_attention(b.q, b.k_cache, b.v_cache)
    kv.check()
    s = torch.cuda.Stream()
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    offsets, lens, pages = b.offsets.clone(), b.kv_lens.clone(), b.pages.contiguous().clone()
    stream = s.cuda_stream if how == "raw" else s
    torch.cuda.synchronize()
    kv.plan(offsets, lens, pages, b.t, stream=stream)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(SLEEP)
    if how == "current":
        with torch.cuda.stream(s):
            kv.paged_attention(b.q, b.k_cache, b.v_cache, out=out)
    else:
        kv.paged_attention(b.q, b.k_cache, b.v_cache, out=out, stream=stream)
    kv.plan(b.offsets, b.kv_lens, b.pages, b.t, stream=stream)
    like = pages.shape
    del offsets, lens, pages
    others = [torch.zeros(like, dtype=torch.int32, device=DEV) for _ in range(4)]  # (a page that there is)
    torch.cuda.synchronize()
    kv.check()
    assert torch.equal(out, want) and all(bool((x == 0).all()) for x in others)
    kv.close()


def test_unaligned_arrays_of_whole_numbers_are_refused():
    b = Batch([3], [40], 4, 2, 64, 16).fill()
    kv = b.handle()
    arrays = [b.offsets, b.kv_lens, b.pages]
    good = kv.paged_attention(b.q, b.k_cache, b.v_cache)
    for i, by in ((0, 4), (0, 1), (1, 2), (2, 2), (2, 1)):
        at = [x.data_ptr() for x in arrays]
        at[i] += by
        with pytest.raises(pkg.SmetricError):
            pkg.smetric_kv_plan(kv.handle, at[0], 1, 3, at[1], at[2], 3, 3)
    q = pkg.smetric_heads(b.q.data_ptr(), 4 * 64, 64)
    for by in (1, 2, 3):
        with pytest.raises(pkg.SmetricError):
            pkg.smetric_qk_norm_rope(kv.handle, q, pkg.smetric_heads(), b.kv_lens.data_ptr() + by, 1, pkg.smetric_kv_transform(), q,
                                     pkg.smetric_heads())
    kv.check()
    assert torch.equal(kv.paged_attention(b.q, b.k_cache, b.v_cache), good)  # the plan stands
    kv.close()
