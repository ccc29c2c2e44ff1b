"""Cases of the paged KV$ operators with the cache in 4 bits: append, read, paged_attention.

A serving instance that holds its KV$ blocks in 4 bits keeps three and a half
times as many of them: the chunk that the prefix hit did not cover is
quantised as it joins the cache, its queries attend over codes and scales, and
blocks are read back in 16 bits where something else wants them. A code is a
sign, two bits of exponent and one of mantissa (0, 0.5, 1, 1.5, 2, 3, 4, 6);
16 elements of a head share a scale of 8 bits (e4m3, the nearest to the largest
magnitude / 6), and a cache a power of two. A case's lengths follow from the
case; its values and the order of its pages follow from the seed."""

import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
GROUP = 16  # elements that share a scale
MOST_FLOPS = 2.4e12  # of a drawn case
MOST_BYTES = 1.2e9
MOST_SCORES = 4.6e9  # entries of the plain form's padded score matrix


def listed():
    heads = dict(heads=32, kv_heads=4, dim=128, k_exp=0, v_exp=0)
    attend = dict(kind="attend", dtype="bf16", page=32, layout="nhd", window=0, lse=False, **heads)
    append = dict(kind="append", dtype="bf16", page=32, layout="nhd", rot=128, interleaved=False, **heads)
    read = dict(kind="read", dtype="bf16", page=32, layout="nhd", **heads)
    return [
        # one decoding step's tokens, one for each of 48 requests, and what the cache then holds for them
        dict(append, name="append_step", n=48, new_lo=1, new_hi=1, ctx_lo=2000, ctx_hi=48000, norm=False, with_q=False, lens=1),
        # the chunks that 16 agent turns append (256 to 4,096 new tokens), with the norms and the queries in the same pass
        dict(append, name="append_turns", n=16, new_lo=256, new_hi=4096, ctx_lo=0, ctx_hi=16000, norm=True, with_q=True, lens=2, page=16),
        # whole prompts into an empty cache: half precision, interleaved rotation of half of each head, heads outside tokens
        dict(append, name="append_prompts", n=5, new_lo=5000, new_hi=32000, ctx_lo=0, ctx_hi=0, norm=False, with_q=False, lens=3,
             dtype="f16", heads=16, kv_heads=8, dim=64, rot=32, interleaved=True, layout="hnd", page=64, v_exp=-3),
        # one request's last 300 positions: latency
        dict(read, name="read_tail", n=1, ctx_lo=24576, ctx_hi=24576, rows_lo=300, rows_hi=300, lens=10),
        # the prefixes of 16 requests, to be handed on in 16 bits
        dict(read, name="read_prefixes", n=16, ctx_lo=2000, ctx_hi=24000, rows_lo=1500, rows_hi=24000, lens=11, dtype="f16", layout="hnd",
             page=64, k_exp=1),
        # one request's single token over a coding agent's mean prompt: latency
        dict(attend, name="decode_one", n=1, new_lo=1, new_hi=1, ctx_lo=24576, ctx_hi=24576, lens=4),
        # a decoding batch of 64 requests with prompts of 2k to 48k tokens: bandwidth
        dict(attend, name="decode_batch", n=64, new_lo=1, new_hi=1, ctx_lo=2000, ctx_hi=48000, lens=5),
        # short conversations, a key head for every query head, half precision, small pages
        dict(attend, name="decode_short", n=19, new_lo=1, new_hi=1, ctx_lo=0, ctx_hi=900, lens=6, dtype="f16", heads=16, kv_heads=16,
             dim=64, page=16, lse=True),
        # 16 query heads for each key head, pages of 128 with heads outside tokens
        dict(attend, name="decode_grouped", n=37, new_lo=1, new_hi=1, ctx_lo=1000, ctx_hi=30000, lens=12, heads=64, layout="hnd", page=128,
             lse=True, k_exp=-2, v_exp=1),
        # turns of 128 to 1,024 new tokens on a prefix hit
        dict(attend, name="chunk_turns", n=8, new_lo=128, new_hi=1024, ctx_lo=2048, ctx_hi=24000, lens=7, page=16),
        # a chunk of a long coding context, blocks of 64
        dict(attend, name="chunk_long", n=1, new_lo=2048, new_hi=2048, ctx_lo=65000, ctx_hi=65000, lens=8, page=64),
        # chunks and single tokens in one batch, requests with nothing new, a sliding window, 7 query heads for each key head
        dict(attend, name="mixed_window", n=24, new_lo=0, new_hi=700, singles=12, ctx_lo=0, ctx_hi=9000, lens=9, dtype="f16", heads=28,
             page=64, window=4096, layout="hnd", lse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        dim = rng.choice([32, 64, 96, 128, 128, 128])
        kv = rng.choice([1, 2, 4, 4, 8, 16])
        case = dict(kind=rng.choice(["append", "append", "read", "attend", "attend", "attend", "attend"]),
                    dtype=rng.choice(["bf16", "bf16", "f16"]), heads=kv * rng.choice([1, 2, 4, 5, 7, 8, 16]), kv_heads=kv, dim=dim,
                    page=rng.choice([16, 32, 64, 128]), layout=rng.choice(["nhd", "nhd", "hnd"]), k_exp=rng.choice([0, 0, -2, 1]),
                    v_exp=rng.choice([0, 0, -3, 2]), lens=rng.randrange(1 << 20))
        if case["heads"] > 64:
            continue
        if case["kind"] == "read":
            rows, hi = _log(rng, 1, 24000), _log(rng, 1, 48000)
            case.update(n=_log(rng, 1, 64), ctx_lo=hi // 8, ctx_hi=hi, rows_lo=rows // 8, rows_hi=rows)
        else:
            style = rng.choice(["step", "turns", "long"])
            if style == "step":
                hi = _log(rng, 16, 48000)
                case.update(n=_log(rng, 1, 256), new_lo=1, new_hi=1, ctx_lo=hi // 16, ctx_hi=hi)
            elif style == "turns":
                new, hi = _log(rng, 2, 4096), _log(rng, 1, 24000)
                n = _log(rng, 1, 24)
                case.update(n=n, new_lo=new // 8, new_hi=new, singles=rng.choice([0, n // 2]), ctx_lo=0, ctx_hi=hi)
            else:
                new, hi = _log(rng, 16, 8192), _log(rng, 1, 65000)
                case.update(n=1, new_lo=new, new_hi=new, ctx_lo=hi, ctx_hi=hi)
            if case["kind"] == "append":
                case.update(rot=rng.choice([dim, dim, 32]), interleaved=rng.random() < 0.3, norm=rng.random() < 0.5, with_q=rng.random() < 0.5)
            else:
                case.update(window=rng.choice([0, 0, 0, _log(rng, 16, 8192)]), lse=rng.random() < 0.5)
        w = work(case)
        if w["flops"] > MOST_FLOPS or w["bytes"] > MOST_BYTES:
            continue
        if case["kind"] == "attend":
            new, kv_lens = _lengths(case)
            if len(new) * case["heads"] * max(new) * max(kv_lens) > MOST_SCORES or case["n"] * max(kv_lens) * kv * dim > 2e9:
                continue
        return case


def _lengths(case):
    """New tokens (or positions read) and length (cached and new) of every request."""
    rng = random.Random(case["lens"])
    if case["kind"] == "read":
        lens = [max(1, rng.randint(case["ctx_lo"], case["ctx_hi"])) for _ in range(case["n"])]
        return [max(1, min(x, rng.randint(case["rows_lo"], case["rows_hi"]))) for x in lens], lens
    new = [1 if i < case.get("singles", 0) else rng.randint(case["new_lo"], case["new_hi"]) for i in range(case["n"])]
    if sum(new) == 0:
        new[0] = 1
    return new, [rng.randint(case["ctx_lo"], case["ctx_hi"]) + x for x in new]


def work(case):
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    new, kv_lens = _lengths(case)
    t, held = sum(new), 2 * hk * (d // 2 + d // GROUP)  # bytes of a token in the cache
    if case["kind"] == "read":
        return {"bytes": t * (held + 2 * hk * d * 2), "flops": t * 2 * hk * d * 2}
    if case["kind"] == "append":  # the heads in, codes and scales out; and those in and the values out again
        q = hq if case["with_q"] else 0
        return {"bytes": t * ((2 * hk + 2 * q) * d * 2 + held + case["rot"] * 4 + 12 + held + 2 * hk * d * 2), "flops": t * (2 * hk * 2 + q) * d * 8}
    window = case["window"] or 1 << 40
    rows = pairs = 0
    for n, kv in zip(new, kv_lens):
        if n == 0:
            continue
        first = kv - n  # position of the first new token
        rows += kv - max(0, first + 1 - window)
        short = min(max(window - 1 - first, 0), n)  # queries that see every key before them
        pairs += short * first + short * (short + 1) // 2 + (n - short) * window
    return {"bytes": t * hq * (d * 4 + (4 if case["lse"] else 0)) + rows * held, "flops": 4 * d * hq * pairs}


def _table(positions, rot, device):
    """cos and sin of every position, side by side."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, device=device, dtype=torch.float64) / rot)
    a = torch.arange(positions, device=device, dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = TYPES[case["dtype"]]
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    normal = lambda *shape: torch.randn(*shape, generator=g, device=dev, dtype=dt)  # noqa: E731
    s = dict(case=case)
    new, kv_lens = _lengths(case)
    n, t, page = case["n"], sum(new), case["page"]
    need = [-(-x // page) for x in kv_lens]
    pool = sum(need) + 8
    order = torch.randperm(pool, generator=g, device=dev).to(torch.int32)
    table = torch.full((n, max(need)), -1, dtype=torch.int32, device=dev)
    held = torch.arange(max(need), device=dev)[None] < torch.tensor(need, device=dev)[:, None]
    table[held] = order[:sum(need)]
    s["pages"] = table
    s["offsets"] = torch.tensor([0] + new, device=dev).cumsum(0)
    s["kv_lens"] = torch.tensor(kv_lens, dtype=torch.int32, device=dev)
    s["first"] = torch.tensor([kv - x for x, kv in zip(new, kv_lens)], dtype=torch.int32, device=dev)
    # codes of two elements a byte, the first in the low four bits; the scales' rows are 4 or 8 bytes wide
    codes, scales = [], []
    for exp in (case["k_exp"], case["v_exp"]):
        shape = (pool, page, hk) if case["layout"] == "nhd" else (pool, hk, page)
        c = torch.empty(*shape, d // 2, dtype=torch.uint8, device=dev)
        w = torch.zeros(*shape, 4 if d <= 64 else 8, dtype=torch.float8_e4m3fn, device=dev)
        part = max(1, (1 << 26) // (page * hk * d))
        for a in range(0, pool, part):
            x = torch.randn(min(part, pool - a), *shape[1:], d, generator=g, device=dev) * 2.0 ** exp
            c[a:a + part], w[a:a + part, ..., :d // GROUP] = _quantise(x, exp)
        as_seen = lambda x: x if case["layout"] == "nhd" else x.transpose(1, 2)  # noqa: E731
        codes.append(as_seen(c))
        scales.append(as_seen(w))
    s["codes"], s["scales"] = codes, scales
    if case["kind"] == "append":
        s["q_norm"], s["k_norm"] = (1 + 0.2 * normal(d).float()).to(dt), (1 + 0.2 * normal(d).float()).to(dt)
        qkv = 2 * normal(t, (hq + 2 * hk) * d)  # a fused projection's output
        s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hk * d, hk * d], 1))
        s["cos_sin"] = _table(max(kv_lens), case["rot"], dev)
        s["q_out"] = torch.empty(t, hq, d, dtype=dt, device=dev)
    elif case["kind"] == "attend":
        s["q"] = 2 * normal(t, hq, d)
    s["dt"], s["rows"] = dt, t
    # where each row's keys and values are, for the plain form
    r = torch.repeat_interleave(torch.arange(n, device=dev), torch.tensor(new, device=dev))
    j = torch.arange(t, device=dev) - s["offsets"][r]
    s["request"], s["place"] = r, j
    s["position"] = s["first"][r] + j
    s["longest_new"], s["longest"] = max(new), max(kv_lens)
    if own:
        import paper_2607_08565_gb300 as pkg
        s["kv"] = pkg.SMetricKV4(head_dim=d, num_q_heads=hq, num_kv_heads=hk, page_size=page, num_pages=pool, max_batch_requests=n,
                                 max_batch_tokens=t, dtype=dt)
        s["cache"] = [pkg.Cache4(c, w, exp) for c, w, exp in zip(codes, scales, (case["k_exp"], case["v_exp"]))]
        # a step's plan, which every layer's calls share
        s["kv"].plan(s["offsets"], s["kv_lens"], s["pages"], t, window=case.get("window", 0))
    return s


def run(s):
    c = s["case"]
    if own:
        kv = s["kv"]
        if c["kind"] == "attend":
            return kv.paged_attention(s["q"], *s["cache"], want_lse=c["lse"])
        if c["kind"] == "append":
            norms = dict(q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS) if c["norm"] else {}
            q = dict(q=s["q"], q_out=s["q_out"]) if c["with_q"] else {}
            kv.append(*s["cache"], s["k"], s["v"], cos_sin=s["cos_sin"], interleaved=c["interleaved"], **norms, **q)
        # what the cache holds at those positions
        values = kv.read(*s["cache"], s["offsets"], s["pages"], s["rows"], first=s["first"])
        return values + (s["q_out"],) if c["kind"] == "append" and c["with_q"] else values
    if c["kind"] == "attend":
        return _attend(s)
    if c["kind"] == "append":
        q = _append(s)
        return _read(s) + ((q,) if c["with_q"] else ())
    return _read(s)


# -- plain forms: elementary operations in 32 bits (64 up to a code's border), rounded once at the end --

def _quantise(x, exp):
    """Codes, two a byte, and scales of heads of values."""
    x = (x * 2.0 ** -exp).unflatten(-1, (-1, GROUP))
    top = x.abs().amax(-1)
    scale = (top / torch.full_like(top, 6)).clamp(max=448).to(torch.float8_e4m3fn)  # (a quotient; by a number it is a product)
    y = x / scale.to(x.dtype)[..., None]
    y = y.nan_to_num(0.0, math.inf, -math.inf)  # (a scale of zero has zeros)
    a = y.abs()
    code = torch.zeros(a.shape, dtype=torch.uint8, device=a.device)
    # borders between the values; one in the middle goes to the code that ends in 0
    for border, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= border) if up else (a > border)
    code += 8 * (y < 0).to(torch.uint8)
    code = code.flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], scale


def _values(codes, scales, exp):
    """The values of rows of codes and scales, in 32 bits."""
    levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    levels = torch.cat([levels, -levels])
    x = torch.stack([levels[(codes & 15).long()], levels[(codes >> 4).long()]], -1).flatten(-2)
    used = scales[..., :x.shape[-1] // GROUP].float() * 2.0 ** exp
    return (x.unflatten(-1, (-1, GROUP)) * used[..., None]).flatten(-2)


def _transform(s, x, weight):
    c = s["case"]
    x = x.double()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.double()
    rot = c["rot"]
    row = s["cos_sin"].double()[s["position"].long()][:, None]
    cos, sin = row[..., :rot // 2], row[..., rot // 2:]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    y, z = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([y, z], -1).flatten(-2) if c["interleaved"] else torch.cat([y, z], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _slots(s):
    page = s["case"]["page"]
    return s["pages"][s["request"], s["position"] // page].long(), s["position"] % page


def _append(s):
    c = s["case"]
    at, slot = _slots(s)
    used = c["dim"] // GROUP
    heads = (_transform(s, s["k"], s["k_norm"] if c["norm"] else None), s["v"].double())
    for x, codes, scales, exp in zip(heads, s["codes"], s["scales"], (c["k_exp"], c["v_exp"])):
        code, scale = _quantise(x, exp)
        codes[at, slot] = code
        scales.view(torch.uint8)[..., :used][at, slot] = scale.view(torch.uint8)
    return _transform(s, s["q"], s["q_norm"] if c["norm"] else None).to(s["dt"]) if c["with_q"] else None


def _read(s):
    at, slot = _slots(s)
    exps = s["case"]["k_exp"], s["case"]["v_exp"]
    return tuple(_values(codes[at, slot], scales.view(torch.uint8)[at, slot].view(torch.float8_e4m3fn), exp).to(s["dt"])
                 for codes, scales, exp in zip(s["codes"], s["scales"], exps))


def _attend(s):
    c = s["case"]
    n, hq, hk, d = c["n"], c["heads"], c["kv_heads"], c["dim"]
    keys = torch.arange(s["longest"], device=s["q"].device)
    held = keys[None] < s["kv_lens"][:, None]
    at, slot = s["pages"][:, keys // c["page"]].long().clamp(min=0), keys % c["page"]

    def gather(i):
        scales = s["scales"][i].view(torch.uint8)[at, slot].view(torch.float8_e4m3fn)
        x = _values(s["codes"][i][at, slot], scales, (c["k_exp"], c["v_exp"])[i])
        return x.masked_fill_(~held[..., None, None], 0.0).permute(0, 2, 1, 3)

    q = torch.zeros(n, s["longest_new"], hq, d, device=s["q"].device)
    q[s["request"], s["place"]] = s["q"].float()
    q = q.unflatten(2, (hk, hq // hk)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # requests, key heads, tokens x group
    x = torch.matmul(q, gather(0).transpose(2, 3)).mul_(d ** -0.5)
    new = s["offsets"][1:] - s["offsets"][:-1]
    pos = (s["kv_lens"] - new)[:, None] + torch.arange(s["longest_new"], device=x.device)
    seen = (keys <= pos[..., None]) & held[:, None]
    if c["window"]:
        seen &= keys > pos[..., None] - c["window"]
    seen = seen.repeat_interleave(hq // hk, 1)[:, None]
    x.masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x, gather(1)) / total.clamp(min=1e-30)
    back = lambda y: y.unflatten(2, (-1, hq // hk)).permute(0, 2, 1, 3, 4).flatten(2, 3)[s["request"], s["place"]]  # noqa: E731
    o = back(o).to(s["dt"])
    return (o, back(total.log() + top)[..., 0]) if c["lse"] else o


# -- the definitions in 64 bits --

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    new, kv_lens = _lengths(case)
    page, d = case["page"], case["dim"]
    exps = (case["k_exp"], case["v_exp"])
    pages = s["pages"].long()
    where = [torch.arange(kv - n, kv, device=pages.device) for n, kv in zip(new, kv_lens)]
    if case["kind"] == "read":
        return tuple(torch.cat([_decoded(s, i, pages[r, p // page], p % page) * 2.0 ** exp for r, p in enumerate(where)])
                     for i, exp in enumerate(exps))
    if case["kind"] == "append":
        p = torch.cat(where)
        k = _turned(case, s["k"], s["k_norm"] if case["norm"] else None, p, s)
        out = (_nearest(k, exps[0]), _nearest(s["v"].double(), exps[1]))
        return out + ((_turned(case, s["q"], s["q_norm"] if case["norm"] else None, p, s),) if case["with_q"] else ())
    group = case["heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=s["q"].device)
    first = 0
    for r, (n, kv) in enumerate(zip(new, kv_lens)):
        if n == 0:
            continue
        j = torch.arange(kv, device=out.device)
        k, v = (_decoded(s, i, pages[r, j // page], j % page) * 2.0 ** exp for i, exp in enumerate(exps))
        for h in range(case["heads"]):
            for a in range(0, n, 2048):
                b = min(n, a + 2048)
                p = torch.arange(kv - n + a, kv - n + b, device=out.device)[:, None]
                hidden = (j > p) | ((j <= p - case["window"]) if case["window"] else False)
                x = (s["q"][first + a:first + b, h].double() @ k[:, h // group].T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                lse[first + a:first + b, h] = torch.logsumexp(x, -1)
                out[first + a:first + b, h] = torch.softmax(x, -1) @ v[:, h // group]
        first += n
    return (out, lse) if case["lse"] else out


def _decoded(s, i, page, slot):
    """Codes and scales at slots of pages, bit by bit: (-1)^sign 2^(e-1) (1 + m/2), or m/2 where e is 0; scales of 4 and 3 bits alike."""
    b = s["codes"][i][page, slot].long()
    b = torch.stack([b % 16, b // 16], -1).flatten(-2)
    e, m = b // 2 % 4, (b % 2).double()
    x = torch.where(e > 0, (1 + m / 2) * _power(e - 1), m / 2) * (1 - 2 * (b // 8)).double()
    w = s["scales"][i].view(torch.uint8)[page, slot][..., :x.shape[-1] // GROUP].long()
    e, m = w // 8 % 16, (w % 8).double()
    w = torch.where(e > 0, (1 + m / 8) * _power(e - 7), m / 8 * 2.0 ** -6) * (1 - 2 * (w // 128)).double()
    return (x.unflatten(-1, (-1, GROUP)) * w[..., None]).flatten(-2)


def _power(e):
    """2 ** e in 64 bits, put together from its bits."""
    return ((e + 1023) << 52).view(torch.float64)


def _nearest(x, exp):
    """What is left of values in 64 bits after they were held in 4."""
    x = (x * 2.0 ** -exp).unflatten(-1, (-1, GROUP))
    top = x.abs().amax(-1, keepdim=True)
    want = (top / torch.full_like(top, 6)).clamp(max=448)
    step = _power(torch.frexp(want)[1].clamp(min=-5).long() - 4)  # between scales there
    scale = torch.round(want / step) * step  # (halves to even)
    y = torch.where(scale > 0, x / scale, 0.0)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6)
    return (a * y.sign() * scale * 2.0 ** exp).flatten(-2)


def _turned(case, x, weight, pos, s):
    """The norm and the rotation, pair by pair as complex numbers."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / case["dim"] + EPS) * weight.double()
    rot = case["rot"]
    row = s["cos_sin"].double()[pos]
    turn = torch.complex(row[:, :rot // 2], row[:, rot // 2:])[:, None]
    pairs = x[..., :rot].unflatten(-1, (rot // 2, 2)) if case["interleaved"] else x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y = y.flatten(-2) if case["interleaved"] else y.transpose(-1, -2).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)
