"""Plain 64-bit forms of the paged KV$ operators and batches to test them on."""

from __future__ import annotations

import torch

import paper_2607_08565_gb300 as pkg

DEV = torch.device("cuda:0")
BF, HF = torch.bfloat16, torch.float16
UNIT = {BF: 2.0 ** -8, HF: 2.0 ** -11}  # largest relative error of one rounding
TINY = {BF: 2.0 ** -134, HF: 2.0 ** -25}  # and its largest absolute error below the normal range


def table(rows, rot):
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    a = torch.arange(rows, dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float().to(DEV)


def transform64(x, weight, pos, cos_sin, interleaved, eps):
    """The norm and rotation in 64 bits: (values, the sum of magnitudes that each is made of)."""
    x = x.double()
    if weight is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    y, mag = x.clone(), x.abs()
    if cos_sin is not None:
        rot = cos_sin.shape[1]
        c, s = (cos_sin.double()[pos.long(), None, i * rot // 2:(i + 1) * rot // 2] for i in (0, 1))
        i = torch.arange(rot // 2, device=x.device)
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        a, b = x[..., p], x[..., q]
        y[..., p], y[..., q] = a * c - b * s, b * c + a * s
        mag[..., p], mag[..., q] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, mag


def assert_close(got, want, mag, dtype, ctx=""):
    """One rounding to dtype of a 32-bit computation whose terms' magnitudes sum to mag."""
    tol = UNIT[dtype] * want.abs() + 2.0 ** -18 * mag + TINY[dtype]
    off = (got.double() - want).abs() - tol
    assert got.isfinite().all() and (off <= 0).all(), f"{ctx}: {int((off > 0).sum())} values off, by {off.max():.3g}"


class Batch:
    """A batch of requests (new tokens, length) over a paged cache whose unused
    slots and unused pages hold `junk`."""

    def __init__(self, new, lens, hq, hk, d, page, dtype=BF, layout="nhd", seed=0, junk=float("nan"), window=0, gap=(0, 0),
                 spare_pages=3, peak=1.0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.new, self.lens, self.hq, self.hk, self.d, self.page, self.dtype, self.window = new, lens, hq, hk, d, page, dtype, window
        self.n, self.first = len(new), gap[0]
        self.t = sum(new) + sum(gap)
        need = [-(-x // page) for x in lens]
        self.pool = sum(need) + spare_pages
        order = torch.randperm(self.pool, generator=g, device=DEV).to(torch.int32)
        most = max(need + [1])
        self.pages = torch.full((self.n, most + 2), -7, dtype=torch.int32, device=DEV)[:, :most]  # rows wider than used
        at = 0
        for r, k in enumerate(need):
            self.pages[r, :k] = order[at:at + k]
            at += k
        rnd = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dtype)  # noqa: E731
        self.keys, self.values = [rnd(x, hk, d) for x in lens], [rnd(x, hk, d) for x in lens]
        shape = {"nhd": (self.pool, page, hk, d), "hnd": (self.pool, hk, page, d), "pair": (self.pool, 2, page, hk, d)}[layout]
        if layout == "pair":
            both = torch.full(shape, junk, dtype=dtype, device=DEV)
            self.k_cache, self.v_cache = both[:, 0], both[:, 1]
        else:
            see = (lambda c: c) if layout == "nhd" else (lambda c: c.transpose(1, 2))
            self.k_cache, self.v_cache = (see(torch.full(shape, junk, dtype=dtype, device=DEV)) for _ in range(2))
        self.offsets = torch.tensor([gap[0]] + new, device=DEV, dtype=torch.int64).cumsum(0)
        self.kv_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.q = peak * torch.randn(self.t, hq, d, generator=g, device=DEV)
        self.q = self.q.to(dtype)

    def slots(self, r, lo=0, hi=None):
        p = torch.arange(lo, self.lens[r] if hi is None else hi, device=DEV)
        return self.pages[r].long()[p // self.page], p % self.page

    def fill(self):
        """Puts every request's keys and values into the cache (what no query sees stays junk)."""
        for r in range(self.n):
            lo = max(0, self.lens[r] - self.new[r] - self.window + 1) if self.window and self.new[r] else 0
            pg, sl = self.slots(r, lo)
            self.k_cache[pg, sl] = self.keys[r][lo:]
            self.v_cache[pg, sl] = self.values[r][lo:]
        return self

    def handle(self, max_requests=None, max_tokens=None):
        kv = pkg.SMetricKV(self.d, self.hq, self.hk, self.page, self.pool, max_requests or max(self.n, 1),
                           max_tokens or max(self.t, 1), dtype=self.dtype)
        kv.plan(self.offsets, self.kv_lens, self.pages, self.t, window=self.window)
        return kv

    def attend64(self, scale=None):
        """(out, lse, sum of p |v|) in 64 bits."""
        scale = self.d ** -0.5 if scale is None else scale
        out = torch.zeros(self.t, self.hq, self.d, dtype=torch.float64, device=DEV)
        mag, lse = out.clone(), torch.full((self.t, self.hq), -float("inf"), dtype=torch.float64, device=DEV)
        a = self.first
        for r in range(self.n):
            b, group = a + self.new[r], self.hq // self.hk
            if self.new[r]:
                k = self.keys[r].double().repeat_interleave(group, 1)
                v = self.values[r].double().repeat_interleave(group, 1)
                x = torch.einsum("thd,khd->htk", self.q[a:b].double(), k) * scale
                pos = torch.arange(self.lens[r] - self.new[r], self.lens[r], device=DEV)[:, None]
                j = torch.arange(self.lens[r], device=DEV)[None]
                hidden = j > pos
                if self.window:
                    hidden = hidden | (j <= pos - self.window)
                x = x.masked_fill(hidden, -float("inf"))
                p = x.softmax(-1)
                out[a:b] = torch.einsum("htk,khd->thd", p, v)
                mag[a:b] = torch.einsum("htk,khd->thd", p, v.abs())
                lse[a:b] = x.logsumexp(-1).T
            a = b
        return out, lse, mag

    def assert_attends(self, out, lse=None, scale=None, ctx=""):
        """The 32-bit softmax, its weights rounded once to the cache's type, the
        output rounded once. A score of magnitude s has an error of about
        (d + 2) 2^-24 s and moves its weight by as much, 2^-12 for s below 30."""
        want, wl, mag = self.attend64(scale)
        u = UNIT[self.dtype]
        tol = u * want.abs() + (u + 2.0 ** -12) * mag + TINY[self.dtype]
        off = (out.double() - want).abs() - tol
        assert out.isfinite().all(), f"{ctx}: not finite"
        assert (off <= 0).all(), f"{ctx}: {int((off > 0).sum())} of {off.numel()} values off, by {off.max():.3g}"
        if lse is not None:
            none = wl.isinf()
            assert torch.equal(lse.isinf(), none), f"{ctx}: rows without keys"
            err = (lse.double() - wl)[~none].abs()
            assert (err <= 2.0 ** -12).all(), f"{ctx}: lse off by {err.max():.3g}"
