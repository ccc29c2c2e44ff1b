"""Caches in 4 bits in 64-bit arithmetic: what quantising gives, what codes and
scales stand for, and batches whose requests are held so."""

from __future__ import annotations

import torch

import paper_2607_08565_gb300 as pkg
from kv_util import BF, DEV, Batch

GROUP = 16
# what the numbers of either type stand for, by their bits without the sign
LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
SCALES = torch.tensor([(8 + b % 8) * 2.0 ** (b // 8 - 10) if b >= 8 else b * 2.0 ** -9 for b in range(127)], dtype=torch.float64)


def nearest(x, numbers):
    """Index of the number nearest to x >= 0, of two alike the even one."""
    numbers = numbers.to(x.device)
    i = (torch.searchsorted(numbers, x.contiguous(), right=True) - 1).clamp(0, len(numbers) - 2)
    below, above = x - numbers[i], numbers[i + 1] - x
    return torch.where((above < below) | ((above == below) & (i % 2 == 1)), i + 1, i)


def quantise64(x, exp=0):
    """(codes [..., D], bits of the scales [..., D / 16]) of heads of finite values."""
    y = (x.double() * 2.0 ** -exp).unflatten(-1, (-1, GROUP))
    top = y.abs().amax(-1)
    bits = nearest(top / torch.full_like(top, 6), SCALES)
    s = SCALES.to(x.device)[bits][..., None]
    codes = nearest(torch.where(s > 0, y.abs() / s, 0.0), LEVELS)
    return (codes + 8 * ((y < 0) & (codes > 0))).flatten(-2), bits


def values64(codes, bits, exp=0):
    """What codes [..., D] and bits of scales [..., D / 16] stand for."""
    s = SCALES.to(codes.device)
    s = torch.cat([s, torch.full_like(s[:1], float("nan")), -s, torch.full_like(s[:1], float("nan"))])[bits.long()]
    x = LEVELS.to(codes.device)[codes.long() % 8] * (1 - 2 * (codes.long() // 8))
    return (x.unflatten(-1, (-1, GROUP)) * s[..., None]).flatten(-2) * 2.0 ** exp


def packed(codes):
    codes = codes.to(torch.uint8)
    return codes[..., 0::2] + 16 * codes[..., 1::2]


def unpacked(b):
    return torch.stack([b % 16, b // 16], -1).flatten(-2)


def scale_row(d):
    return 4 if d <= 64 else 8


class Batch4(Batch):
    """A batch over caches in 4 bits. Unused slots and pages hold codes of any
    kind and scales that are NaN. keys and values become what is held of them."""

    def __init__(self, *args, exps=(0, 0), layout="nhd", **kw):
        super().__init__(*args, **kw)
        self.exps = exps
        g = torch.Generator(device=DEV)
        g.manual_seed(kw.get("seed", 0) + 1)
        dims = (self.pool, self.page, self.hk)
        self.caches = []
        both = None
        for i, exp in enumerate(exps):
            widths = self.d // 2, scale_row(self.d)
            if layout == "nhd":
                made = [torch.empty(*dims, w, dtype=torch.uint8, device=DEV) for w in widths]
            elif layout == "hnd":
                made = [torch.empty(self.pool, self.hk, self.page, w, dtype=torch.uint8, device=DEV).transpose(1, 2) for w in widths]
            else:  # "pair": keys and values of a page side by side, rows with room between them
                if both is None:
                    both = [torch.empty(self.pool, 2, self.page, self.hk + 1, w + 16, dtype=torch.uint8, device=DEV) for w in widths]
                made = [x[:, i, :, 1:, :w] for x, w in zip(both, widths)]
            made[0].copy_(torch.randint(0, 256, made[0].shape, generator=g, device=DEV, dtype=torch.uint8))
            made[1].fill_(0x7F)
            self.caches.append(pkg.Cache4(made[0], made[1].view(torch.float8_e4m3fn), exp))
        self.held = [[quantise64(x, e) for x in xs] for xs, e in zip((self.keys, self.values), exps)]
        self.keys, self.values = ([values64(*h, e) for h in held] for held, e in zip(self.held, exps))

    def bytes_of(self, i):
        """Codes and scales of a cache, as bytes."""
        c = self.caches[i]
        return c.codes, c.scales.view(torch.uint8)

    def fill(self):
        for r in range(self.n):
            lo = max(0, self.lens[r] - self.new[r] - self.window + 1) if self.window and self.new[r] else 0
            pg, sl = self.slots(r, lo)
            for i in range(2):
                codes, scales = self.bytes_of(i)
                codes[pg, sl] = packed(self.held[i][r][0][lo:])
                scales[..., :self.d // GROUP][pg, sl] = self.held[i][r][1][lo:].to(torch.uint8)
        return self

    def handle(self, max_requests=None, max_tokens=None):
        kv = pkg.SMetricKV4(self.d, self.hq, self.hk, self.page, self.pool, max_requests or max(self.n, 1),
                            max_tokens or max(self.t, 1), dtype=self.dtype)
        kv.plan(self.offsets, self.kv_lens, self.pages, self.t, window=self.window)
        return kv


__all__ = ["BF", "DEV", "GROUP", "LEVELS", "SCALES", "Batch4", "nearest", "packed", "quantise64", "scale_row", "unpacked", "values64"]
