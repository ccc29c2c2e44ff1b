"""Edges of the operators over the 4-bit paged cache: rows and pages that are not
numbers or not there, sizes at the ends of their ranges, other streams, captured
calls, and the calls together as a serving instance makes them."""

import importlib.util
import os

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv4_util import DEV, GROUP, Batch4, packed, quantise64, scale_row, values64
from kv_util import BF, HF, UNIT, table

pytestmark = pytest.mark.gpu
SLEEP = 200_000_000  # cycles: about 0.1 s, longer than the host takes to go on


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def check(b, scale=None):
    kv = b.handle()
    out, lse = kv.paged_attention(b.q, *b.caches, scale=scale, want_lse=True)
    kv.check()
    b.assert_attends(out, lse, scale)
    kv.close()
    return out, lse


@pytest.mark.parametrize("hq,hk,d,new,lens", [
    (8, 2, 64, [1, 1], [100, 3]),             # nobody shares them
    (8, 2, 64, [300], [300]),                 # two tiles of queries
    (64, 64, 128, [1], [24577]),
    (16, 1, 96, [1], [24577]),                # 152 pieces
    (16, 2, 128, [40], [30000]),              # of many rows
])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_a_nan_query_stays_nan(hq, hk, d, new, lens, dtype):
    b = Batch4(new, lens, hq, hk, d, 64, dtype, seed=hk).fill()
    kv = b.handle()
    good, good_lse = kv.paged_attention(b.q, *b.caches, want_lse=True)
    kv.check()
    b.assert_attends(good, good_lse)
    for token, head in ((0, 0), (b.t - 1, hq - 1), (b.t // 2, hq // 2)):
        q = b.q.clone()
        q[token, head, d // 2] = float("nan")
        out, lse = kv.paged_attention(q, *b.caches, want_lse=True)
        kv.check()
        assert bool(out[token, head].isnan().all()) and bool(lse[token, head].isnan())
        out[token, head], lse[token, head] = good[token, head], good_lse[token, head]
        assert torch.equal(out, good) and torch.equal(lse, good_lse)
    kv.close()


@pytest.mark.parametrize("new,lens", [([1, 1], [3000, 70]), ([200, 3], [900, 70])])
@pytest.mark.parametrize("power", [-100, -30, 30, 100])
def test_queries_of_any_size(new, lens, power):
    """Queries times a power of two, scores divided by it: the same outputs, bit for bit. And rows of sizes of their own."""
    b = Batch4(new, lens, 16, 2, 128, 32).fill()
    kv = b.handle()
    good, good_lse = kv.paged_attention(b.q, *b.caches, want_lse=True)
    out, lse = kv.paged_attention(b.q * 2.0 ** power, *b.caches, scale=128 ** -0.5 * 2.0 ** -power, want_lse=True)
    kv.check()
    assert torch.equal(out, good) and torch.equal(lse, good_lse)
    kv.close()
    b.q = b.q * (2.0 ** torch.randint(-12, 2, b.q.shape[:2], device=DEV))[..., None].to(BF)
    check(b)


@pytest.mark.parametrize("new,lens", [([1, 1], [3000, 70]), ([200, 3], [900, 70])])
def test_queries_up_to_the_largest(new, lens):
    """Rows whose largest elements are in the type's last power of two. (None so small that half precision
    would round it: the same outputs, bit for bit, as of the rows divided by 2^126.)"""
    b = Batch4(new, lens, 16, 2, 128, 32).fill()
    b.q = b.q.clamp(-3.5, 3.5) * (b.q.abs() > 2.0 ** -8)
    b.q[:, :, 5] = 3.0
    kv = b.handle()
    good, good_lse = kv.paged_attention(b.q, *b.caches, scale=1.0, want_lse=True)
    kv.check()
    # Scores of up to 40: their errors of (d + 2) 2^-24 each are within 2^-11 of a weight; weights below 2^-21 of the
    # largest are off by up to 2^-32 of it (half precision's smallest step), each with its value.
    want, want_lse, mag = b.attend64(1.0)
    values = torch.stack([b.values[r].abs().sum(0) for r in range(b.n) for _ in range(b.new[r])]).repeat_interleave(8, 1)
    off = (good.double() - want).abs() - (2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -32 * values)
    assert bool((off <= 0).all()) and bool(((good_lse.double() - want_lse).abs() <= 2.0 ** -11).all())
    big = b.q * 2.0 ** 126
    assert bool((big.abs().amax(-1) >= 2.0 ** 127).all()) and bool(big.isfinite().all())
    out, lse = kv.paged_attention(big, *b.caches, scale=2.0 ** -126, want_lse=True)
    kv.check()
    kv.close()
    assert torch.equal(out, good) and torch.equal(lse, good_lse)


@pytest.mark.parametrize("window", [100, 400])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("new", [1, 3, 40])
def test_the_longest_sequence(window, dtype, new):
    """A request of 2^31 - 1 tokens, of which a window is seen; scales that are NaN past its end and before the window."""
    d, page, kv_len, group = 32, 256, 2 ** 31 - 1, 4
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    pages = torch.full((1, 2 ** 31 // page), -7, dtype=torch.int32, device=DEV)
    pages[0, -3:] = torch.tensor([1, 2, 3], dtype=torch.int32)
    kv = pkg.SMetricKV4(d, group, 1, page, 5, 1, new, dtype=dtype)
    caches = kv.new_cache()
    last = 3 * page - 1  # places in the three pages, in a row: the one past the end
    first = last - new - window + 1
    held = []
    for c in caches:
        codes, bits = quantise64(torch.randn(window + new - 1, 1, d, generator=g, device=DEV).to(dtype))
        c.scales.view(torch.uint8).fill_(0x7F)
        c.codes[1:4].view(3 * page, 1, d // 2)[first:last] = packed(codes)
        c.scales.view(torch.uint8)[1:4].view(3 * page, 1, 4)[first:last, :, :d // GROUP] = bits.to(torch.uint8)
        held.append(values64(codes, bits)[:, 0])
    q = torch.randn(new, group, d, generator=g, device=DEV).to(dtype)
    kv.plan(torch.tensor([0, new], device=DEV), torch.tensor([kv_len], dtype=torch.int32, device=DEV), pages, new, window=window)
    out, lse = kv.paged_attention(q, *caches, want_lse=True)
    kv.check()
    for i in range(new):
        keys, values = (x[i:i + window] for x in held)
        x = q[i].double() @ keys.T * d ** -0.5
        p = x.softmax(-1)
        want, mag = p @ values, p @ values.abs()
        u = UNIT[dtype]  # (the bound that the other attention tests use)
        assert bool(((out[i].double() - want).abs() <= u * want.abs() + (u + 2.0 ** -12) * mag).all())
        assert bool(((lse[i].double() - x.logsumexp(-1)).abs() <= 2.0 ** -12).all())
    # appended there, and read back
    k = torch.randn(new, 1, d, generator=g, device=DEV).to(dtype)
    kv.append(*caches, k, k)
    got, _ = kv.read(caches[0], None, torch.tensor([0, new], device=DEV), pages, new,
                     first=torch.tensor([kv_len - new], dtype=torch.int32, device=DEV))
    kv.check()
    assert torch.equal(got.double(), values64(*quantise64(k)))
    kv.close()


def test_caches_past_32_bits():
    """Codes and scales more than 2^32 bytes from the cache's start."""
    d, hk, page = 128, 8, 256
    pool = 2 ** 32 // (page * hk * 8) + 40  # scales of 4.3 GB, codes of 34
    kv = pkg.SMetricKV4(d, 2 * hk, hk, page, pool, 2, 400)
    caches = kv.new_cache()
    lens, new = [700, 300], [300, 1]
    pages = torch.tensor([[pool - 1, 3, pool - 2], [pool - 9, 5, -1]], dtype=torch.int32, device=DEV)
    b = Batch4(new, lens, 2 * hk, hk, d, page)
    for i, c in enumerate(caches):
        for r in range(2):
            at = torch.arange(lens[r], device=DEV)
            p, s = pages[r].long()[at // page], at % page
            c.codes[p, s] = packed(b.held[i][r][0])
            c.scales.view(torch.uint8)[p, s] = b.held[i][r][1].to(torch.uint8)
    kv.plan(b.offsets, b.kv_lens, pages, b.t)
    out, lse = kv.paged_attention(b.q, *caches, want_lse=True)
    kv.check()
    b.assert_attends(out, lse)
    kv.plan(torch.tensor([0, 1, 2], device=DEV), b.kv_lens, pages, 2)  # single tokens
    out = kv.paged_attention(b.q[[299, 300]], *caches)
    kv.check()
    b.new, b.t, b.q = [1, 1], 2, b.q[[299, 300]]
    b.assert_attends(out)
    k, v = kv.read(*caches, torch.tensor([0] + lens, device=DEV).cumsum(0), pages, sum(lens))
    assert torch.equal(k.double(), torch.cat(b.keys)) and torch.equal(v.double(), torch.cat(b.values))
    x = torch.randn(2, hk, d, device=DEV).to(BF)
    kv.append(*caches, x, x)
    k, _ = kv.read(caches[0], None, torch.tensor([0, 1, 2], device=DEV), pages, 2, first=b.kv_lens - 1)
    kv.check()
    assert torch.equal(k.double(), values64(*quantise64(x)))
    kv.close()


@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 5]])
@pytest.mark.parametrize("page", [16, 128])
def test_pages_that_are_not_there(new, page):
    """Their keys and values are zeros, and the error is latched."""
    b = Batch4(new, [300, 200, 150], 8, 2, 128, page).fill()
    bad = [(0, 0, -5), (1, 100 // page, b.pool), (2, 140 // page, 2 ** 31 - 1)]
    for r, i, page_number in bad:
        b.pages[r, i] = page_number
        lo, hi = i * page, min((i + 1) * page, b.lens[r])
        b.keys[r][lo:hi] = 0
        b.values[r][lo:hi] = 0
    kv = b.handle()
    assert kv.status() in (pkg.SMETRIC_OK, pkg.SMETRIC_ERR_INVALID_ARG)  # (a new token's page latches in the plan)
    out, lse = kv.paged_attention(b.q, *b.caches, want_lse=True)
    assert kv.status() == pkg.SMETRIC_ERR_INVALID_ARG and kv.status() == pkg.SMETRIC_OK
    b.assert_attends(out, lse)
    kv.close()


@pytest.mark.parametrize("hq,hk", [(13, 13), (24, 24), (50, 25), (120, 8), (16, 16), (12, 12), (17, 1), (100, 1)])
def test_numbers_of_heads(hq, hk):
    """More key heads than a CTA has warps, and more query heads a key head than single tokens have rows."""
    d = 64
    check(Batch4([1] * 4, [2000, 1, 77, 300], hq, hk, d, 32, gap=(2, 1)).fill())
    check(Batch4([0, 70, 1, 2], [20, 400, 33, 300], hq, hk, d, 32, gap=(1, 3)).fill())


def test_chunks_among_as_many_requests_as_tokens():
    """More requests than tokens, some of which have several: all go the way of single tokens."""
    for new in ([5, 0, 0, 0, 0, 1, 0], [0, 40] + [0] * 50, [0, 0, 0, 3]):
        lens = [x + 17 * (i % 5) + 30 for i, x in enumerate(new)]
        for hq, hk, d in ((8, 2, 128), (6, 6, 32), (16, 1, 64)):
            check(Batch4(new, lens, hq, hk, d, 16, gap=(0, 0)).fill())
            check(Batch4(new, lens, hq, hk, d, 16, window=20).fill())


def test_no_tokens_and_no_requests():
    b = Batch4([0, 0], [5, 40], 4, 2, 64, 16, gap=(3, 0)).fill()
    out, lse = check(b)
    assert (out == 0).all() and lse.isinf().all()
    kv = pkg.SMetricKV4(64, 4, 2, 16, 3, 0, 4)
    none = torch.zeros(1, dtype=torch.int64, device=DEV)
    kv.plan(none, none[:0].int(), torch.zeros(0, 2, dtype=torch.int32, device=DEV), 4)
    q = torch.ones(4, 4, 64, dtype=BF, device=DEV)
    out, lse = kv.paged_attention(q, *kv.new_cache(), want_lse=True)
    kv.check()
    assert (out == 0).all() and lse.isinf().all()
    kv.plan(none, none[:0].int(), torch.zeros(0, 2, dtype=torch.int32, device=DEV), 0)
    assert kv.paged_attention(q[:0], *kv.new_cache()).shape == (0, 4, 64)
    kv.close()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("d,dtype", [(32, BF), (64, BF), (96, HF), (128, HF), (128, BF)])
@pytest.mark.parametrize("requests,new", [(1, 1), (120, 1), (3, 20)])
def test_each_page_is_read_in_its_place(page, d, dtype, requests, new):
    """Keys of one length and queries along one of them each: its score is 4 sqrt(d), 22 or more, above most others', so
    that the output is its value but for weights of a few thousandths in all; requests share the pages."""
    length, group = 6001, 4
    g = torch.Generator(device=DEV)
    g.manual_seed(page + d)
    used = -(-length // page)
    pool = used + 3
    order = torch.randperm(pool, generator=g, device=DEV)[:used]
    kv = pkg.SMetricKV4(d, group, 1, page, pool, requests, requests * new, dtype=dtype)
    caches = kv.new_cache()
    at = torch.arange(length, device=DEV)
    held = []
    for c in caches:
        x = torch.randn(length, 1, d, generator=g, device=DEV)
        codes, bits = quantise64(x * (d ** 0.5 / x.norm(dim=-1, keepdim=True)))
        c.scales.view(torch.uint8).fill_(0x7F)
        c.codes[order[at // page], at % page] = packed(codes)
        c.scales.view(torch.uint8)[order[at // page], at % page] = torch.nn.functional.pad(
            bits, (0, scale_row(d) - d // GROUP), value=0x7F).to(torch.uint8)
        held.append(values64(codes, bits)[:, 0])
    t = requests * new
    kv.plan(torch.arange(requests + 1, device=DEV) * new, torch.full((requests,), length, dtype=torch.int32, device=DEV),
            order.to(torch.int32).repeat(requests, 1), t)
    targets = torch.linspace(0, used - 1, t * group, device=DEV).round().long()
    targets = (targets * page + targets * 7 % page).clamp(max=length - new).view(t, group)
    q = (4 * held[0][targets]).to(dtype)
    out = kv.paged_attention(q, *caches)
    kv.check()
    last = length - new + torch.arange(new, device=DEV).repeat(requests)
    x = torch.einsum("tgd,kd->tgk", q.double(), held[0]) * d ** -0.5
    x = x.masked_fill(at[None, None] > last[:, None, None], -float("inf"))
    p = x.softmax(-1)
    want, mag = p @ held[1], p @ held[1].abs()
    # Scores of up to 4 sqrt(d) * 1.2: their errors of (d + 2) 2^-24 each are within 2^-11 of a weight. Weights are
    # rounded to half precision, the row's largest being 2^7 or more: those below 2^-14 are off by up to half of its
    # smallest step, 2^-25, which is 2^-32 of the largest and so of their sum, each of them with its value. (A value of
    # zero at the key that is singled out leaves nothing but such weights.)
    u = UNIT[dtype]
    tol = u * want.abs() + (u + 2.0 ** -11) * mag + 2.0 ** -32 * held[1].abs().sum(0)
    off = (out.double() - want).abs() - tol
    assert bool((off <= 0).all()), f"{int((off > 0).sum())} values off, by {off.max():.3g}"
    kv.close()


def test_a_captured_step_replayed():
    """Plan, append, attention and reading back in a graph, with other inputs in its tensors."""
    new, lens = [1, 40, 1, 3], [300, 700, 65, 40]
    b = Batch4(new, lens, 16, 2, 128, 32).fill()
    kv = b.handle()
    k, v = (torch.randn(b.t, 2, 128, device=DEV).to(BF) for _ in range(2))
    cs = table(1000, 128)
    rows = torch.tensor([0] + lens, device=DEV).cumsum(0)

    def step():
        kv.plan(b.offsets, b.kv_lens, b.pages, b.t)
        q = kv.append(*b.caches, k, v, q=b.q, cos_sin=cs)
        return kv.paged_attention(q, *b.caches, want_lse=True) + kv.read(*b.caches, rows, b.pages, sum(lens))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = step()
    for seed in range(3):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        for x in (k, v, b.q):
            x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        if seed == 2:  # other lengths too
            b.kv_lens -= torch.tensor([3, 30, 0, 2], dtype=torch.int32, device=DEV)
        graph.replay()
        torch.cuda.synchronize()
        kv.check()
        held = [x.clone() for x in got]
        with torch.cuda.stream(s):
            again = step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, again))
    kv.close()


def _calls(kv, b, stream):
    k, v = (torch.cat([x[-n:] for x, n in zip(xs, b.new)]).to(b.dtype) for xs in (b.keys, b.values))
    rows = torch.tensor([0] + b.lens, device=DEV).cumsum(0)
    torch.cuda.synchronize()
    return [
        lambda: list(kv.paged_attention(b.q, *b.caches, want_lse=True, stream=stream)),
        lambda: [kv.append(*b.caches, k, v, q=b.q, stream=stream)],
        lambda: list(kv.read(*b.caches, rows, b.pages, sum(b.lens), stream=stream)),
    ]


@pytest.mark.parametrize("raw", [False, True])
def test_new_outputs_on_another_stream(raw):
    """Their memory is not handed out again before that stream has written it,
    nor written before the current stream is done with its last owner."""
    b = Batch4([40, 1], [300, 70], 8, 2, 64, 16).fill()
    s = torch.cuda.Stream()
    kv = b.handle()
    for call in _calls(kv, b, s.cuda_stream if raw else s):
        got = call()
        torch.cuda.synchronize()
        like = [x.clone() for x in got]
        del got
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        with torch.cuda.stream(s):
            torch.cuda._sleep(SLEEP)
        call()  # dropped before they are written
        others = [torch.full_like(x, 7.0) for x in like for _ in range(2)]
        torch.cuda.synchronize()
        assert all(bool((x == 7).all()) for x in others)
        del others
        torch.cuda.empty_cache()
        owners = [torch.full_like(x, 3.0) for x in like for _ in range(2)]  # whose memory is still being read
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


def test_two_handles_at_once():
    """On two streams, over the same cache."""
    b = Batch4([1, 130, 1], [3000, 800, 70], 16, 2, 128, 32).fill()
    one, two = b.handle(), b.handle()
    want = one.paged_attention(b.q, *b.caches)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [kv.paged_attention(b.q, *b.caches, stream=s) for kv, s in zip((one, two), streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, want) for x in got)
    one.check(), two.check()
    one.close(), two.close()


def test_calls_of_the_other_kind_are_refused():
    four, wide = pkg.SMetricKV4(64, 4, 2, 16, 3, 2, 8), pkg.SMetricKV(64, 4, 2, 16, 3, 2, 8)
    plan = (torch.tensor([0, 4], device=DEV), torch.tensor([20], dtype=torch.int32, device=DEV), torch.zeros(1, 2, dtype=torch.int32, device=DEV), 4)
    four.plan(*plan), wide.plan(*plan)
    k4, v4 = (four._cache4(c, "") for c in four.new_cache())
    k16 = torch.zeros(3, 16, 2, 64, dtype=BF, device=DEV)
    c16 = wide._cache(k16, k16.clone())
    q, k = torch.zeros(4, 4, 64, dtype=BF, device=DEV), torch.zeros(4, 2, 64, dtype=BF, device=DEV)
    qh, kh, no, t = four._heads(q, 4, 4, ""), four._heads(k, 2, 4, ""), pkg.smetric_heads(), pkg.smetric_kv_transform()
    for call in (lambda: pkg.smetric_kvq_append(wide.handle, k4, v4, kh, kh, no, no, t),
                 lambda: pkg.smetric_kvq_attention(wide.handle, k4, v4, qh, 1.0, qh),
                 lambda: pkg.smetric_kvq_read(wide.handle, k4, v4, plan[0], 1, 4, None, plan[2], 2, 2, kh, kh),
                 lambda: pkg.smetric_kv_append(four.handle, c16, kh, kh, no, no, t),
                 lambda: pkg.smetric_paged_attention(four.handle, c16, qh, 1.0, qh)):
        with pytest.raises(pkg.SmetricError):
            call()
    # the transform alone is both kinds'
    pos = torch.arange(4, dtype=torch.int32, device=DEV)
    kw = dict(cos_sin=table(10, 64), q_norm=torch.ones(64, dtype=BF, device=DEV), k_norm=torch.ones(64, dtype=BF, device=DEV))
    q.normal_(), k.normal_()
    assert all(torch.equal(x, y) for x, y in zip(four.qk_norm_rope(q, k, pos, **kw), wide.qk_norm_rope(q, k, pos, **kw)))
    four.check(), wide.check()
    four.close(), wide.close()


def test_bad_descriptions_are_refused():
    kv = pkg.SMetricKV4(128, 4, 2, 16, 3, 2, 8)
    kv.plan(torch.tensor([0, 4], device=DEV), torch.tensor([20], dtype=torch.int32, device=DEV), torch.zeros(1, 2, dtype=torch.int32, device=DEV), 4)
    cache = kv.new_cache()
    q, k = torch.zeros(4, 4, 128, dtype=BF, device=DEV), torch.zeros(4, 2, 128, dtype=BF, device=DEV)
    qh, kh, no, t = kv._heads(q, 4, 4, ""), kv._heads(k, 2, 4, ""), pkg.smetric_heads(), pkg.smetric_kv_transform()
    good = kv._cache4(cache[0], "")
    fields = [f for f, _ in good._fields_]
    bad = [("d_codes", 8), ("d_codes", None), ("d_scales", 4), ("d_scales", None), ("page_stride", 8), ("token_stride", 24), ("head_stride", 40),
           ("page_stride", -16), ("scale_page_stride", 4), ("scale_token_stride", 12), ("scale_head_stride", 2), ("exp", 65), ("exp", -65),
           ("reserved", 1), ("page_stride", 2 ** 32), ("token_stride", 2 ** 33), ("scale_page_stride", 2 ** 32), ("scale_token_stride", 2 ** 40)]
    offsets, pages = torch.tensor([0, 4], device=DEV), torch.zeros(1, 2, dtype=torch.int32, device=DEV)
    for name, value in bad:
        values = {f: getattr(good, f) for f in fields}
        values[name] = value if name[:2] != "d_" or value is None else values[name] + value
        c = pkg.smetric_kvq_cache(*values.values())
        for k4, v4 in ((c, good), (good, c)):
            for call in (lambda: pkg.smetric_kvq_append(kv.handle, k4, v4, kh, kh, no, no, t),
                         lambda: pkg.smetric_kvq_attention(kv.handle, k4, v4, qh, 1.0, qh),
                         lambda: pkg.smetric_kvq_read(kv.handle, k4, v4, offsets, 1, 4, None, pages, 2, 2, kh, kh)):
                with pytest.raises(pkg.SmetricError):
                    call()
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(pkg.SmetricError):
            kv.paged_attention(q, *cache, scale=scale)
    with pytest.raises(pkg.SmetricError):  # scale * 2^exp past 32 bits
        kv.paged_attention(q, cache[0]._replace(exp=64), cache[1], scale=1e30)
    for args in (dict(n=-1), dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(most=-1), dict(stride=1), dict(offsets=None), dict(pages=None),
                 dict(offsets=offsets.data_ptr() + 4), dict(pages=pages.data_ptr() + 2), dict(first=pages.data_ptr() + 1)):
        a = dict(n=1, n_rows=4, most=2, stride=2, offsets=offsets, pages=pages, first=None)
        a.update(args)
        with pytest.raises(pkg.SmetricError):
            pkg.smetric_kvq_read(kv.handle, good, good, a["offsets"], a["n"], a["n_rows"], a["first"], a["pages"], a["most"], a["stride"], kh, kh)
    kv.check()
    assert bool((cache[0].codes == 0).all())
    kv.close()


def test_steps_of_a_conversation():
    """A prompt, then single tokens and short chunks: what each attends over is what was quantised, all of it read back."""
    hq, hk, d, page, dtype = 16, 2, 128, 16, BF
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    b = Batch4([1, 1], [400, 300], hq, hk, d, page, dtype)
    kv = b.handle(max_requests=2, max_tokens=400)
    done = [0, 0]
    kept = [[], []]
    for new in ([150, 60], [1, 1], [1, 1], [0, 40], [1, 3], [70, 1], [1, 1]):
        t = sum(new)
        q, k, v = (torch.randn(t, h, d, generator=g, device=DEV).to(dtype) for h in (hq, hk, hk))
        lens = [x + n for x, n in zip(done, new)]
        offsets = torch.tensor([0] + new, device=DEV).cumsum(0)
        kv.plan(offsets, torch.tensor(lens, dtype=torch.int32, device=DEV), b.pages, t)
        kv.append(*b.caches, k, v)
        for r in range(2):
            kept[r].append((k[offsets[r]:offsets[r + 1]], v[offsets[r]:offsets[r + 1]]))
        out, lse = kv.paged_attention(q, *b.caches, want_lse=True)
        kv.check()
        b.new, b.lens, b.t, b.q = new, lens, t, q
        b.keys, b.values = ([values64(*quantise64(torch.cat([x[i] for x in kept[r]]))) for r in range(2)] for i in range(2))
        b.assert_attends(out, lse, ctx=str(new))
        done = lens
    k, v = kv.read(*b.caches, torch.tensor([0] + done, device=DEV).cumsum(0), b.pages, sum(done))
    kv.check()
    assert torch.equal(k.double(), torch.cat(b.keys)) and torch.equal(v.double(), torch.cat(b.values))
    kv.close()


def test_turns_on_cached_blocks():
    """The routing and serving example with its caches in 4 bits: prompts prefilled on a prefix hit give the outputs
    that they give from nothing."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    spec = importlib.util.spec_from_file_location("serve_turns", os.path.join(root, "examples", "serve_turns.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    done, total, worst = ex.serve(sessions=10, turns=3, instances=2, say=lambda *_: None, bits=4)
    assert done < total // 2
    # the same codes and scales: a few roundings of outputs below 4 apart
    assert worst <= 8 * 2.0 ** -8 * 4
