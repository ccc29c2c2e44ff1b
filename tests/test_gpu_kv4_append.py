"""Quantising keys and values as they join the 4-bit paged cache, and reading
them back, against 64-bit forms; what the calls do not own stays as it was."""

import pytest
import torch

import paper_2607_08565_gb300 as pkg
from kv4_util import DEV, GROUP, LEVELS, SCALES, Batch4, nearest, packed, quantise64, unpacked, values64
from kv_util import BF, HF, assert_close, table, transform64

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def bits(x):
    return x.contiguous().view(torch.uint8)


def same(a, b):
    return torch.equal(bits(a), bits(b))


def assert_nearest(codes, scales, y, err, exp, ctx):
    """codes [.., D] and scale bits are nearest to 32-bit values that are within err of y."""
    y, err = y * 2.0 ** -exp, err * 2.0 ** -exp
    y, err = y.unflatten(-1, (-1, GROUP)), err.unflatten(-1, (-1, GROUP))
    top, off = y.abs().amax(-1), err.amax(-1)
    table_s, table_c = SCALES.to(y.device), LEVELS.to(y.device)
    want = (top / torch.full_like(top, 6)).clamp(max=448)
    assert (scales < 127).all(), f"{ctx}: a NaN or a sign in the scales"
    s = table_s[scales.long()]
    # (a division rounded to 32 bits, and the values' errors)
    slack = off / 6 + 2.0 ** -22 * want
    assert ((s - want).abs() <= (table_s[nearest(want, SCALES)] - want).abs() + 2 * slack).all(), f"{ctx}: scales"
    c = codes.unflatten(-1, (-1, GROUP))
    got = table_c[c.long() % 8] * (1 - 2 * (c.long() // 8)) * s[..., None]
    best = (table_c[nearest(torch.where(s[..., None] > 0, y.abs() / s[..., None], 0.0), LEVELS)] * s[..., None] - y.abs()).abs()
    # (quotients rounded to multiples of 2^-19, 2^-20 off at most, after a product 2^-20 off)
    assert ((got - y).abs() <= best + 2 * (err + 2.0 ** -19 * s[..., None])).all(), f"{ctx}: codes"


def run_append(b, rot, interleaved, q_norm, k_norm, with_q, in_place=False, eps=1e-6, seed=99):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    qkv = (3 * torch.randn(b.t, (b.hq + 2 * b.hk) * b.d, generator=g, device=DEV)).to(b.dtype)
    q, k, v = (x.unflatten(1, (-1, b.d)) for x in qkv.split([b.hq * b.d, b.hk * b.d, b.hk * b.d], 1))
    cs = table(max(b.lens + [1]), rot) if rot else None
    wq, wk = ((1 + 0.3 * torch.randn(b.d, generator=g, device=DEV)).to(b.dtype) for _ in range(2))
    wq, wk = wq if q_norm else None, wk if k_norm else None
    before = [[x.clone() for x in b.bytes_of(i)] for i in range(2)]
    before_q = q.clone()
    kv = b.handle()
    q_out = (q if in_place else torch.full((b.t, b.hq, b.d), 5.0, dtype=b.dtype, device=DEV)) if with_q else None
    kv.append(*b.caches, k, v, q=q if with_q else None, q_out=q_out, cos_sin=cs, interleaved=interleaved, q_norm=wq, k_norm=wk, eps=eps)
    kv.check()
    owned = torch.zeros(b.pool, b.page, dtype=torch.bool, device=DEV)
    a, used = b.first, b.d // GROUP
    for r in range(b.n):
        e, lo = a + b.new[r], b.lens[r] - b.new[r]
        pg, sl = b.slots(r, lo)
        owned[pg, sl] = True
        pos = torch.arange(lo, b.lens[r], device=DEV)
        kc, ks = (x[pg, sl] for x in b.bytes_of(0))
        y, mag = transform64(k[a:e], wk, pos, cs, interleaved, eps)
        moved = wk is not None or cs is not None
        assert_nearest(unpacked(kc), ks[..., :used], y, 2.0 ** -18 * mag * moved, b.exps[0], f"keys of request {r}")
        vc, vs = (x[pg, sl] for x in b.bytes_of(1))
        codes, scales = quantise64(v[a:e], b.exps[1])
        assert torch.equal(vs[..., :used].long(), scales), f"scales of the values of request {r}"
        got = unpacked(vc).long()
        assert torch.equal(got * (got != 8), codes), f"codes of the values of request {r}"  # (zeros of either sign)
        if with_q:
            y, mag = transform64(before_q[a:e], wq, pos, cs, interleaved, eps)
            assert_close(q_out[a:e], y, mag, b.dtype, f"queries of request {r}")
        a = e
    for i in range(2):
        for now, was in zip(b.bytes_of(i), before[i]):
            assert torch.equal(now[~owned], was[~owned])
        assert torch.equal(b.bytes_of(i)[1][..., used:], before[i][1][..., used:])  # the scales' unused bytes
    if with_q and not in_place:  # tokens of no request
        assert (q_out[:b.first] == 5).all() and (q_out[a:] == 5).all()
    kv.close()


MIX = ([1, 0, 7, 33, 1, 64, 0, 130], [1, 0, 40, 33, 65, 64, 17, 300])


@pytest.mark.parametrize("hq,hk,d", [(4, 4, 128), (32, 4, 128), (7, 1, 64), (10, 2, 96), (3, 3, 32), (64, 8, 32), (5, 5, 96)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_append_head_layouts(hq, hk, d, dtype):
    for k, (rot, il) in enumerate([(d, False), (d, True), (16, False), (d - 16, False), (0, False)]):
        b = Batch4(*MIX, hq, hk, d, 16, dtype, seed=k, exps=((0, 0), (2, -1), (-3, 3), (0, 1), (-1, 0))[k])
        run_append(b, rot, il, k % 2 == 0, k < 2, k != 2, in_place=k == 1)


@pytest.mark.parametrize("rot", range(16, 129, 16))
@pytest.mark.parametrize("k_norm", [False, True])
def test_append_rotations_of_part_of_a_head(rot, k_norm):
    """Halves of 8 elements and odd multiples: groups whose pieces two lanes hold."""
    for il in (False, True):
        run_append(Batch4([5, 40], [9, 77], 4, 2, 128, 16), rot, il, False, k_norm, False)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["nhd", "hnd", "pair"])
def test_append_pages_and_strides(page, layout):
    run_append(Batch4(*MIX, 8, 2, 64, page, layout=layout, gap=(3, 5)), 64, False, True, True, True)


def test_append_only_some_norms_and_one_token():
    for qn, kn in [(True, False), (False, True)]:
        run_append(Batch4(*MIX, 4, 2, 96, 32), 32, False, qn, kn, True)
    run_append(Batch4([1], [1], 8, 1, 128, 16), 128, False, True, True, True)
    run_append(Batch4([0, 0], [5, 0], 8, 1, 128, 16), 128, False, True, True, True)


def test_append_many_requests_and_one_long():
    rng = torch.Generator().manual_seed(3)
    new = torch.randint(0, 5, (3000,), generator=rng).tolist()
    lens = [x + int(y) for x, y in zip(new, torch.randint(0, 60, (3000,), generator=rng))]
    b = Batch4(new, lens, 4, 2, 64, 16)
    b.new, b.lens = new, lens
    run_append(b, 64, False, False, True, True)
    run_append(Batch4([20011], [20030], 4, 1, 64, 64), 64, True, True, True, True)


def appended(x, d, dtype, exp=0):
    """Values put into an empty cache: (handle, batch, codes, scale bits) of the values' cache."""
    t = x.shape[0]
    b = Batch4([t], [t], 1, 1, d, 16, dtype, exps=(exp, exp))
    kv = b.handle()
    x = x.to(dtype)[:, None]
    kv.append(*b.caches, x, x)
    kv.check()
    pg, sl = b.slots(0)
    for i in range(2):  # keys without a transform are quantised like values
        codes, scales = (y[pg, sl, 0] for y in b.bytes_of(i))
        if i:
            assert same(codes, was[0]) and same(scales, was[1])
        was = codes, scales
    return kv, b, unpacked(codes), scales[:, :d // GROUP]


@pytest.mark.parametrize("dtype", [BF, HF])
def test_every_border_between_codes(dtype):
    """Quotients halfway between two codes, and the nearest ones of the type on both sides, under every scale that
    16-bit values can give exactly so."""
    rows = []
    for byte in range(8, 127):
        s = SCALES[byte].item()
        x = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]) * s
        low, high = (torch.nextafter(x.to(dtype), torch.tensor(z, dtype=dtype)).float() for z in (0.0, INF))
        low[0] = high[0] = x[0]
        rows += [torch.cat([x, -x]), torch.cat([low, -high]), torch.cat([high, -low])]
    x = torch.stack(rows).to(DEV)
    x = torch.cat([x, x.flip(0)], 1)  # two groups: heads of 32
    x = x[(x.abs() <= 60000).all(1)].to(dtype)
    kv, b, codes, scales = appended(x, 32, dtype)
    want, want_s = quantise64(x)
    assert torch.equal(scales.long(), want_s)
    assert torch.equal(codes.long() * (codes != 8), want)
    kv.close()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("exp", [0, -5, 7])
def test_every_border_between_scales(dtype, exp):
    """Largest magnitudes whose sixth is halfway between two scales, and beside; scales that are subnormal or 0, and
    groups past the largest."""
    top = torch.cat([SCALES, (SCALES[1:] + SCALES[:-1]) / 2, torch.tensor([449.0, 464.0, 500.0, 2.0 ** -11, 2.0 ** -12])]) * 6 * 2.0 ** exp
    x = top.to(dtype)
    x = torch.cat([x, torch.nextafter(x, torch.zeros_like(x)), torch.nextafter(x, torch.full_like(x, INF))]).to(DEV)
    x = x[x.isfinite()]
    ramp = torch.linspace(-1, 1, 15, device=DEV)
    x = torch.cat([x[:, None].float(), x[:, None].float() * ramp], 1).to(dtype)
    x = torch.cat([x, -x.flip(0)], 1)
    kv, b, codes, scales = appended(x, 32, dtype, exp)
    want, want_s = quantise64(x, exp)
    assert torch.equal(scales.long(), want_s)
    assert torch.equal(codes.long() * (codes != 8), want)
    kv.close()


@pytest.mark.parametrize("dtype", [BF, HF])
def test_zeros_nan_and_infinities(dtype):
    x = torch.randn(6, 64, device=DEV)
    x[0] = 0
    x[1, 20] = NAN
    x[2, 40] = INF
    x[3, 41] = -INF
    x[4, 3], x[4, 5] = NAN, INF
    x[5, :16] = 1e-30 if dtype == BF else 6e-8  # too small for a scale
    kv, b, codes, scales = appended(x, 64, dtype)
    k, v = kv.read(*b.caches, b.offsets, b.pages, 6)
    kv.check()
    assert same(k, v)
    v = v[:, 0].double()
    assert (v[0] == 0).all() and (scales[0] == 0).all() and (v[5, :16] == 0).all()
    for row, group in ((1, 1), (4, 0)):
        assert v[row, 16 * group:16 * group + 16].isnan().all()
    assert v[2, 40] == 2688 and v[3, 41] == -2688
    bad = torch.zeros(6, 64, dtype=torch.bool, device=DEV)
    bad[1, 16:32] = bad[4, :16] = True
    assert v[~bad].isfinite().all()
    fine = torch.ones(6, 4, dtype=torch.bool, device=DEV)
    fine[1, 1] = fine[4, 0] = fine[2, 2] = fine[3, 2] = False
    want, want_s = quantise64(x.to(dtype).double().nan_to_num(0, 0, 0))
    assert torch.equal(v.unflatten(1, (4, 16))[fine], values64(want, want_s).unflatten(1, (4, 16))[fine])
    kv.close()


def test_large_exponents():
    x = torch.randn(8, 64, device=DEV)
    for exp in (-64, 64):
        kv, b, codes, scales = appended(x * 2.0 ** exp, 64, BF, exp)
        want, want_s = quantise64((x * 2.0 ** exp).to(BF), exp)
        assert torch.equal(scales.long(), want_s) and torch.equal(codes.long() * (codes != 8), want)
        _, v = kv.read(None, b.caches[1], b.offsets, b.pages, 8)
        assert torch.equal(v[:, 0].double(), values64(want, want_s, exp))
        kv.close()


# ---- reading back ----

def read64(b, i, r, lo, n):
    return (b.keys if i == 0 else b.values)[r][lo:lo + n]


@pytest.mark.parametrize("hk,d", [(1, 32), (4, 128), (3, 96), (16, 64), (1, 128)])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("layout", ["nhd", "hnd", "pair"])
def test_read_positions(hk, d, dtype, layout):
    lens = [1, 17, 0, 300, 64, 129, 1000, 5]
    first = [0, 3, 0, 299, 0, 128, 37, 5]
    rows = [1, 14, 0, 1, 64, 1, 900, 0]
    b = Batch4([0] * len(lens), lens, hk, hk, d, 16, dtype, layout=layout, exps=(2, -1)).fill()
    kv = b.handle()
    before, after = 3, 4
    offsets = torch.tensor([before] + rows, device=DEV).cumsum(0)
    n = before + sum(rows) + after
    outs = [torch.full((n, hk, d), 5.0, dtype=dtype, device=DEV) for _ in range(2)]
    got = kv.read(*b.caches, offsets, b.pages, n, first=torch.tensor(first, dtype=torch.int32, device=DEV), k_out=outs[0], v_out=outs[1])
    kv.check()
    for i in range(2):
        assert got[i] is outs[i]
        want = torch.cat([read64(b, i, r, f, m) for r, (f, m) in enumerate(zip(first, rows))])
        assert torch.equal(outs[i][before:n - after].double(), want.to(dtype).double())  # 6 bits: exact in both types
        assert torch.equal(want.to(dtype).double(), want)
        assert (outs[i][:before] == 5).all() and (outs[i][n - after:] == 5).all()
    kv.close()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_read_whole_sequences_of_a_plan(page):
    lens = [700, 1, 15, 16, 17, 255, 256, 257]
    b = Batch4([1] * len(lens), lens, 8, 2, 128, page).fill()
    kv = b.handle()
    offsets = torch.tensor([0] + lens, device=DEV).cumsum(0)
    k, v = kv.read(*b.caches, offsets, b.pages, sum(lens))
    kv.check()
    assert torch.equal(k.double(), torch.cat(b.keys)) and torch.equal(v.double(), torch.cat(b.values))
    k2, none = kv.read(b.caches[0], None, offsets, b.pages, sum(lens))
    none2, v2 = kv.read(None, b.caches[1], offsets, b.pages, sum(lens))
    assert none is None and none2 is None and same(k, k2) and same(v, v2)
    assert kv.read(None, None, offsets, b.pages, sum(lens)) == (None, None)
    kv.close()


def test_read_into_views_and_rounding():
    """Outputs that are part of wider rows; values past half precision's range."""
    b = Batch4([1], [40], 2, 2, 64, 16, HF, exps=(9, 0)).fill()
    b.caches[0].scales.view(torch.uint8).fill_(126)  # 448
    kv = b.handle()
    wide = torch.full((40, 4, 72), 5.0, dtype=HF, device=DEV)
    out = wide[:, 1:3, 8:]
    offsets = torch.tensor([0, 40], device=DEV)
    kv.read(b.caches[0], None, offsets, b.pages, 40, k_out=out)
    kv.check()
    pg, sl = b.slots(0)
    want = values64(unpacked(b.caches[0].codes[pg, sl]), torch.full((40, 2, 4), 126, device=DEV), 9)
    assert torch.equal(out, want.to(HF)) and out.isinf().any()
    assert (wide[:, 0] == 5).all() and (wide[:, 3] == 5).all() and (wide[..., :8] == 5).all()
    kv.close()


def test_read_bad_pages_and_positions_are_zeros():
    b = Batch4([1, 1, 1], [40, 40, 40], 2, 2, 64, 16).fill()
    kv = b.handle()
    pages = b.pages.clone()
    pages[0, 1], pages[1, 0] = -1, b.pool
    offsets = torch.tensor([0, 40, 80, 120], device=DEV)
    k, v = kv.read(*b.caches, offsets, pages, 120)
    assert kv.status() == pkg.SMETRIC_ERR_INVALID_ARG and kv.status() == pkg.SMETRIC_OK
    for got, want in ((k, b.keys), (v, b.values)):
        want = torch.cat(want)
        want[16:32] = 0
        want[40:56] = 0
        assert torch.equal(got.double(), want)
    # before the first position, and past the row of pages (48 tokens)
    k, _ = kv.read(*b.caches, offsets, b.pages, 120, first=torch.tensor([-3, 0, 20], dtype=torch.int32, device=DEV))
    assert kv.status() == pkg.SMETRIC_ERR_INVALID_ARG
    assert (k[:3] == 0).all() and torch.equal(k[3:40].double(), b.keys[0][:37])
    assert torch.equal(k[40:80].double(), b.keys[1]) and torch.equal(k[80:100].double(), b.keys[2][20:]) and (k[108:] == 0).all()
    kv.close()


@pytest.mark.parametrize("offsets", [[0, 50, 40, 120], [0, 40, 80, 121], [-1, 40, 80, 120]])
def test_read_bad_offsets_are_latched(offsets):
    b = Batch4([1, 1, 1], [40, 40, 40], 2, 2, 64, 16).fill()
    kv = b.handle()
    kv.read(*b.caches, torch.tensor(offsets, device=DEV), b.pages, 120)
    assert kv.status() == pkg.SMETRIC_ERR_INVALID_ARG
    kv.close()


def test_read_nothing():
    b = Batch4([1], [40], 2, 2, 64, 16).fill()
    kv = b.handle()
    one = torch.zeros(1, dtype=torch.int64, device=DEV)
    k, v = kv.read(*b.caches, one, b.pages[:0], 0)
    assert k.shape == (0, 2, 64) and v.shape == (0, 2, 64)
    out = torch.full((3, 2, 64), 5.0, dtype=BF, device=DEV)
    kv.read(b.caches[0], None, one, b.pages[:0], 3, k_out=out)
    kv.check()
    assert (out == 5).all()
    kv.close()


def test_append_then_read_is_what_was_held():
    """A chunk, then single tokens, read back as a whole."""
    d, hk, page, dtype = 128, 2, 16, BF
    total = 100
    b = Batch4([60], [total], 4, hk, d, page, dtype)
    kv = b.handle()
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    k, v = (torch.randn(total, hk, d, generator=g, device=DEV).to(dtype) for _ in range(2))
    at = 0
    for n in [60] + [1] * 40:
        kv.plan(torch.tensor([0, n], device=DEV), torch.tensor([at + n], dtype=torch.int32, device=DEV), b.pages, n)
        kv.append(*b.caches, k[at:at + n], v[at:at + n])
        at += n
    gk, gv = kv.read(*b.caches, torch.tensor([0, total], device=DEV), b.pages, total)
    kv.check()
    for got, x in ((gk, k), (gv, v)):
        assert torch.equal(got.double(), values64(*quantise64(x)))
        # within a sixth of the group's largest
        top = x.double().unflatten(-1, (-1, GROUP)).abs().amax(-1, keepdim=True).expand(-1, -1, -1, GROUP).flatten(-2)
        assert ((got.double() - x.double()).abs() <= top / 6 * (1 + 2.0 ** -4)).all()
    assert torch.equal(packed(unpacked(b.caches[0].codes)), b.caches[0].codes)
    kv.close()
