"""A paged cache of 8-bit blocks from its definition, in Python's doubles and lists of the 128 numbers that e4m3 has from 0 on."""
import math

import torch

from history_ref import Cache

# the numbers from 0 on (4 of exponent, 3 of mantissa; the largest code is NaN), and the borders between them
NUMBERS = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)]
BORDERS = [(a + b) / 2 for a, b in zip(NUMBERS, NUMBERS[1:])]
NAN = float("nan")


def nearest(x):
    """The nearest of the numbers in 64 bits, of two equally near the one with the even code; at most 448; NaN stays."""
    values, borders = (torch.tensor(t, dtype=torch.float64, device=x.device) for t in (NUMBERS, BORDERS))
    x = x.double()
    at = torch.searchsorted(borders, x.abs().contiguous())
    tie = borders[at.clamp(max=len(BORDERS) - 1)] == x.abs()
    y = torch.copysign(values[(at + (tie & (at % 2 == 1))).clamp(max=len(NUMBERS) - 1)], x)
    return torch.where(torch.isnan(x), NAN, y)


def needed(x):
    """Exponent of the smallest power of two, within the scale's range, of which 448 cover all finite elements of x."""
    finite = x.double().abs()[torch.isfinite(x)]
    top = finite.max().item() if finite.numel() else 0.0
    e = -100
    while e < 119 and top > 448.0 * 2.0 ** e:
        e += 1
    return e


class Cache8(Cache):
    """A cache whose users hold `lens` items, put there by the definition, a chunk of `chunk` items after another (all at once where it
    is None); what is not an item holds NaN, in codes and scales."""

    def __init__(self, lens, Hkv, D, page, block, dtype, seed=0, chunk=None, magnitude=None, **kw):
        super().__init__(lens, Hkv, D, page, dtype, seed=seed, **kw)
        self.block = block
        self.codes = [torch.full((self.P, Hkv, page, D), NAN, dtype=torch.float64, device=self.device) for _ in range(2)]
        self.scales = [torch.full((self.P, Hkv, page // block), NAN, dtype=torch.float64, device=self.device) for _ in range(2)]
        for u, n in enumerate(lens):
            if magnitude is not None:
                self.items[u] = tuple((t.float() * magnitude(u, n)).to(dtype) for t in self.items[u])
            step = chunk or max(n, 1)
            for a in range(0, n, step):
                self.append(u, *(t[a:min(a + step, n)] for t in self.items[u]), a)

    def append(self, u, k, v, old):
        """Items old, old + 1, .. of user u become k and v [c,Hkv,D]."""
        n = old + k.shape[0]
        for codes, scales, new in zip(self.codes, self.scales, (k, v)):
            for j0 in range(old // self.block * self.block, n, self.block):
                p, place = self.table[u][j0 // self.page], j0 % self.page
                if not 0 <= p < self.P:
                    continue
                for h in range(new.shape[1]):
                    x = new[max(j0 - old, 0):j0 + self.block - old, h].double()
                    scale, held = 2.0 ** needed(x), max(old - j0, 0)
                    was = scales[p, h, place // self.block].item()
                    if held:
                        scale = max(scale, was)
                        old_rows = codes[p, h, place:place + held]
                        codes[p, h, place:place + held] = nearest(old_rows * (was / scale))
                    codes[p, h, place + held:place + held + x.shape[0]] = nearest(x / scale)
                    scales[p, h, place // self.block] = scale

    def tensors(self):
        """k_cache, v_cache, k_scale, v_scale as the library has them."""
        return (*(c.float().to(torch.float8_e4m3fn) for c in self.codes), *(s.float() for s in self.scales))

    def values(self, u, n):
        """(k, v) [n,Hkv,D] of a user in 64 bits, as the cache holds them."""
        out = []
        for codes, scales in zip(self.codes, self.scales):
            if n == 0:
                out.append(torch.zeros(0, *codes.shape[1::2], dtype=torch.float64, device=self.device))
                continue
            page, place = self.places(u, range(n))
            page = page.clamp(0, self.P - 1)
            out.append(codes[page, :, place] * scales[page, :, torch.div(place, self.block, rounding_mode="floor")][..., None])
        return out


def same(got, want):
    """Equal numbers, NaN where NaN."""
    got, want = got.double(), want.double()
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0)) and math.prod(got.shape) == want.numel()
