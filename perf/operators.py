"""Cases of the paged KV$ operators: qk_norm_rope, kv_append, paged_attention.

The operators are what a serving instance runs on the blocks that the router
sent a request to: the chunk of tokens that the prefix hit did not cover is
normed and rotated, its keys and values join the paged cache, and its queries
attend over the cached prefix and the chunk; later tokens come one at a time.
Pages have the index's block sizes. A case's lengths follow from the case; its
values and the order of its pages follow from the seed."""

import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
MOST_FLOPS = 2.4e12  # of a drawn case
MOST_BYTES = 3.4e9
MOST_SCORES = 4.6e9  # entries of the plain form's padded score matrix


def listed():
    heads = dict(heads=32, kv_heads=4, dim=128)
    attend = dict(kind="attend", dtype="bf16", page=32, layout="nhd", window=0, lse=False, **heads)
    append = dict(kind="append", dtype="bf16", page=32, layout="nhd", rot=128, interleaved=False, **heads)
    norm = dict(kind="norm_rope", dtype="bf16", rot=128, interleaved=False, **heads)
    return [
        # one decoding step's tokens, one for each of 48 requests
        dict(append, name="append_step", n=48, new_lo=1, new_hi=1, ctx_lo=2000, ctx_hi=48000, norm=False, with_q=False, lens=1),
        # the chunks that 16 agent turns append (256 to 4,096 new tokens), with the norms and the queries in the same pass
        dict(append, name="append_turns", n=16, new_lo=256, new_hi=4096, ctx_lo=0, ctx_hi=16000, norm=True, with_q=True, lens=2, page=16),
        # whole prompts into an empty cache: half precision, interleaved rotation of half of each head, heads outside tokens
        dict(append, name="append_prompts", n=5, new_lo=5000, new_hi=32000, ctx_lo=0, ctx_hi=0, norm=False, with_q=False, lens=3,
             dtype="f16", heads=16, kv_heads=8, dim=64, rot=32, interleaved=True, layout="hnd", page=64),
        # a decoding step's queries and keys
        dict(norm, name="norm_step", tokens=37, spread=48000),
        # a prefill batch's, 16 query heads for each key head
        dict(norm, name="norm_prefill", tokens=16001, spread=128000, heads=64),
        # one request's single token over a coding agent's mean prompt: latency
        dict(attend, name="decode_one", n=1, new_lo=1, new_hi=1, ctx_lo=24576, ctx_hi=24576, lens=4),
        # a decoding batch of 64 requests with prompts of 2k to 48k tokens: bandwidth
        dict(attend, name="decode_batch", n=64, new_lo=1, new_hi=1, ctx_lo=2000, ctx_hi=48000, lens=5),
        # short conversations, a key head for every query head, half precision, small pages
        dict(attend, name="decode_short", n=19, new_lo=1, new_hi=1, ctx_lo=0, ctx_hi=900, lens=6, dtype="f16", heads=16, kv_heads=16,
             dim=64, page=16, lse=True),
        # turns of 128 to 1,024 new tokens on a prefix hit
        dict(attend, name="chunk_turns", n=8, new_lo=128, new_hi=1024, ctx_lo=2048, ctx_hi=24000, lens=7, page=16),
        # a chunk of a long coding context, blocks of 64
        dict(attend, name="chunk_long", n=1, new_lo=2048, new_hi=2048, ctx_lo=65000, ctx_hi=65000, lens=8, page=64),
        # chunks and single tokens in one batch, requests with nothing new, a sliding window, 7 query heads for each key head
        dict(attend, name="mixed_window", n=24, new_lo=0, new_hi=700, singles=12, ctx_lo=0, ctx_hi=9000, lens=9, dtype="f16", heads=28,
             page=64, window=4096, layout="hnd", lse=True),
        # whole prompts, nothing cached
        dict(attend, name="prefill", n=2, new_lo=7000, new_hi=8192, ctx_lo=0, ctx_hi=0, lens=10),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        dim = rng.choice([64, 96, 128, 128])
        kv = rng.choice([1, 2, 4, 4, 8, 16])
        case = dict(kind=rng.choice(["append", "norm_rope", "attend", "attend", "attend"]), dtype=rng.choice(["bf16", "bf16", "f16"]),
                    heads=kv * rng.choice([1, 2, 4, 5, 7, 8, 16]), kv_heads=kv, dim=dim)
        if case["heads"] > 64:
            continue
        if case["kind"] != "attend":
            case.update(rot=rng.choice([dim, dim, 32]), interleaved=rng.random() < 0.3)
        if case["kind"] == "norm_rope":
            case.update(tokens=_log(rng, 1, 16001), spread=_log(rng, 16, 128000))
        else:
            case.update(page=rng.choice([16, 32, 64, 128]), layout=rng.choice(["nhd", "nhd", "hnd"]), lens=rng.randrange(1 << 20))
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
                case.update(norm=rng.random() < 0.5, with_q=rng.random() < 0.5)
            else:
                case.update(window=rng.choice([0, 0, 0, _log(rng, 16, 8192)]), lse=rng.random() < 0.5)
        w = work(case)
        if w["flops"] > MOST_FLOPS or w["bytes"] > MOST_BYTES:
            continue
        if case["kind"] == "attend":
            new, kv_lens = _lengths(case)
            if len(new) * case["heads"] * max(new) * max(kv_lens) > MOST_SCORES:
                continue
        return case


def _lengths(case):
    """New tokens and length (cached and new) of every request."""
    rng = random.Random(case["lens"])
    new = [1 if i < case.get("singles", 0) else rng.randint(case["new_lo"], case["new_hi"]) for i in range(case["n"])]
    if sum(new) == 0:
        new[0] = 1
    return new, [rng.randint(case["ctx_lo"], case["ctx_hi"]) + x for x in new]


def work(case):
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "norm_rope":
        t = case["tokens"]
        return {"bytes": t * ((hq + hk) * d * 4 + case["rot"] * 4 + 4), "flops": t * (hq + hk) * d * 8}
    new, kv_lens = _lengths(case)
    t = sum(new)
    if case["kind"] == "append":
        heads = 2 * hk + (hq if case["with_q"] else 0)
        return {"bytes": t * (heads * d * 4 + case["rot"] * 4 + 12), "flops": t * heads * d * 8}
    window = case["window"] or 1 << 40
    rows = pairs = 0
    for n, kv in zip(new, kv_lens):
        if n == 0:
            continue
        first = kv - n  # position of the first new token
        rows += kv - max(0, first + 1 - window)
        short = min(max(window - 1 - first, 0), n)  # queries that see every key before them
        pairs += short * first + short * (short + 1) // 2 + (n - short) * window
    return {"bytes": t * hq * d * 4 + rows * hk * d * 4, "flops": 4 * d * hq * pairs}


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
    if case["kind"] != "attend":
        s["q_norm"], s["k_norm"] = (1 + 0.2 * normal(d).float()).to(dt), (1 + 0.2 * normal(d).float()).to(dt)
    if case["kind"] == "norm_rope":
        t = case["tokens"]
        qkv = 2 * normal(t, (hq + 2 * hk) * d)  # a fused projection's output
        s["q"], s["k"] = qkv[:, :hq * d].unflatten(1, (hq, d)), qkv[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
        s["positions"] = torch.randint(0, case["spread"], (t,), generator=g, device=dev, dtype=torch.int32)
        s["cos_sin"] = _table(case["spread"], case["rot"], dev)
        if own:
            import paper_2607_08565_gb300 as pkg
            s["kv"] = pkg.SMetricKV(head_dim=d, num_q_heads=hq, num_kv_heads=hk, page_size=16, num_pages=1, max_batch_requests=1,
                                    max_batch_tokens=t, dtype=dt)
        return s
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
    shape = (pool, page, hk, d) if case["layout"] == "nhd" else (pool, hk, page, d)
    as_seen = lambda c: c if case["layout"] == "nhd" else c.transpose(1, 2)  # noqa: E731
    s["k_cache"], s["v_cache"] = as_seen(normal(*shape)), as_seen(normal(*shape))
    if case["kind"] == "append":
        qkv = 2 * normal(t, (hq + 2 * hk) * d)
        s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hk * d, hk * d], 1))
        s["cos_sin"] = _table(max(kv_lens), case["rot"], dev)
        s["q_out"] = torch.empty(t, hq, d, dtype=dt, device=dev)
    else:
        s["q"] = 2 * normal(t, hq, d)
    # where each new token's keys and values go, for the plain form
    r = torch.repeat_interleave(torch.arange(n, device=dev), torch.tensor(new, device=dev))
    j = torch.arange(t, device=dev) - s["offsets"][r]
    s["request"], s["place"] = r, j
    s["position"] = s["kv_lens"][r] - (s["offsets"][r + 1] - s["offsets"][r]) + j
    s["longest_new"], s["longest"] = max(new), max(kv_lens)
    if own:
        import paper_2607_08565_gb300 as pkg
        s["kv"] = pkg.SMetricKV(head_dim=d, num_q_heads=hq, num_kv_heads=hk, page_size=page, num_pages=pool, max_batch_requests=n,
                                max_batch_tokens=t, dtype=dt)
        # a step's plan, which every layer's calls share
        s["kv"].plan(s["offsets"], s["kv_lens"], s["pages"], t, window=case.get("window", 0))
    return s


def run(s):
    kind = s["case"]["kind"]
    if own:
        c, kv = s["case"], s["kv"]
        if kind == "norm_rope":
            return kv.qk_norm_rope(s["q"], s["k"], s["positions"], cos_sin=s["cos_sin"], interleaved=c["interleaved"], q_norm=s["q_norm"],
                                   k_norm=s["k_norm"], eps=EPS)
        if kind == "append":
            norms = dict(q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS) if c["norm"] else {}
            q = dict(q=s["q"], q_out=s["q_out"]) if c["with_q"] else {}
            kv.append(s["k_cache"], s["v_cache"], s["k"], s["v"], cos_sin=s["cos_sin"], interleaved=c["interleaved"], **norms, **q)
            return (s["k_cache"], s["v_cache"]) + ((s["q_out"],) if c["with_q"] else ())
        return kv.paged_attention(s["q"], s["k_cache"], s["v_cache"], want_lse=c["lse"])
    if kind == "norm_rope":
        return _transform(s, s["q"], s["q_norm"], s["positions"]), _transform(s, s["k"], s["k_norm"], s["positions"])
    return _append(s) if kind == "append" else _attend(s)


# -- plain forms: elementary operations in 32 bits, rounded once at the end --

def _transform(s, x, weight, positions):
    c, dt = s["case"], x.dtype
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    rot = c["rot"]
    row = s["cos_sin"][positions.long()][:, None]
    cos, sin = row[..., :rot // 2], row[..., rot // 2:]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    y, z = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([y, z], -1).flatten(-2) if c["interleaved"] else torch.cat([y, z], -1)
    return torch.cat([y, x[..., rot:]], -1).to(dt)


def _append(s):
    c = s["case"]
    page, slot = s["position"] // c["page"], s["position"] % c["page"]
    at = s["pages"][s["request"], page].long()
    s["k_cache"][at, slot] = _transform(s, s["k"], s["k_norm"] if c["norm"] else None, s["position"])
    s["v_cache"][at, slot] = s["v"]
    if not c["with_q"]:
        return s["k_cache"], s["v_cache"]
    return s["k_cache"], s["v_cache"], _transform(s, s["q"], s["q_norm"] if c["norm"] else None, s["position"])


def _attend(s):
    c = s["case"]
    n, hq, hk, d = c["n"], c["heads"], c["kv_heads"], c["dim"]
    keys = torch.arange(s["longest"], device=s["q"].device)
    held = keys[None] < s["kv_lens"][:, None]
    at = s["pages"][:, keys // c["page"]].long().clamp(min=0)
    gather = lambda x: torch.where(held[..., None, None], x[at, keys % c["page"]].float(), 0.0).permute(0, 2, 1, 3)  # noqa: E731
    q = torch.zeros(n, s["longest_new"], hq, d, device=s["q"].device)
    q[s["request"], s["place"]] = s["q"].float()
    q = q.unflatten(2, (hk, hq // hk)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # requests, key heads, tokens x group
    x = torch.matmul(q, gather(s["k_cache"]).transpose(2, 3)).mul_(d ** -0.5)
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
    o = torch.matmul(x, gather(s["v_cache"])) / total.clamp(min=1e-30)
    back = lambda y: y.unflatten(2, (-1, hq // hk)).permute(0, 2, 1, 3, 4).flatten(2, 3)[s["request"], s["place"]]  # noqa: E731
    o = back(o).to(s["q"].dtype)
    return (o, back(total.log() + top)[..., 0]) if c["lse"] else o


# -- the definitions in 64 bits --

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "norm_rope":
        pos = s["positions"].long()
        return _turned(case, s["q"], s["q_norm"], pos, s), _turned(case, s["k"], s["k_norm"], pos, s)
    new, kv_lens = _lengths(case)
    page, first, at = case["page"], 0, []
    if case["kind"] == "append":
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        pos = torch.cat([torch.arange(kv - n, kv, device=kc.device) for n, kv in zip(new, kv_lens)])
        k = _turned(case, s["k"], s["k_norm"] if case["norm"] else None, pos, s)
        for r, (n, kv) in enumerate(zip(new, kv_lens)):
            p = pos[first:first + n]
            where = s["pages"][r].long()[p // page]
            kc[where, p % page] = k[first:first + n]
            vc[where, p % page] = s["v"][first:first + n].double()
            first += n
        return (kc, vc) + ((_turned(case, s["q"], s["q_norm"] if case["norm"] else None, pos, s),) if case["with_q"] else ())
    group = case["heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=s["q"].device)
    for n, kv, pages in zip(new, kv_lens, s["pages"].long()):
        if n == 0:
            continue
        j = torch.arange(kv, device=out.device)
        pages = pages[:-(-kv // page)]
        for h in range(case["heads"]):
            k, v = (x[pages, :, h // group].flatten(0, 1)[:kv].double() for x in (s["k_cache"], s["v_cache"]))
            for a in range(0, n, 2048):
                b = min(n, a + 2048)
                p = torch.arange(kv - n + a, kv - n + b, device=out.device)[:, None]
                hidden = (j > p) | ((j <= p - case["window"]) if case["window"] else False)
                x = (s["q"][first + a:first + b, h].double() @ k.T / math.sqrt(case["dim"])).masked_fill(hidden, -math.inf)
                lse[first + a:first + b, h] = torch.logsumexp(x, -1)
                out[first + a:first + b, h] = torch.softmax(x, -1) @ v
        first += n
    return (out, lse) if case["lse"] else out


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
