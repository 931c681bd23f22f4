"""Reference of rotary angles in all their forms and of the cache in blocks, in fp64 / plain Python -- TEST INFRASTRUCTURE ONLY (nothing
in the product path may import this)."""
from __future__ import annotations

import math
from typing import Optional

import numpy as np
import torch

BLOCK, LEAST, MOST = 16, -117, 120


def frequencies(dims: int, base: float, scaling: Optional[str] = None, factor: float = 1.0, context: int = 0, low: float = 1.0, high: float = 32.0):
    if scaling == "base":
        base = base * factor ** (dims / (dims - 2))
    out = []
    for i in range(dims // 2):
        f = base ** (-2.0 * i / dims)
        if scaling == "linear":
            f /= factor
        if scaling == "bands":
            keep = (context * f / (2 * math.pi) - low) / (high - low)
            keep = min(1.0, max(0.0, keep))
            f = keep * f + (1 - keep) * f / factor
        out.append(f)
    return np.array(out)


def turn(x: torch.Tensor, table: torch.Tensor, positions, interleaved: bool, transpose: bool = False) -> torch.Tensor:
    """x [rows, heads, d], table fp32 [n, 2, dims / 2], every product and sum rounded to fp32; rows whose position is None are 0."""
    x, half = x.float().cpu(), table.shape[2]
    out = torch.zeros_like(x)
    for r, p in enumerate(positions):
        if p is None:
            continue
        c, s = table[p, 0].cpu(), table[p, 1].cpu() * (-1.0 if transpose else 1.0)
        out[r] = x[r]
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            xa, xb = x[r, :, a], x[r, :, b]
            out[r, :, a] = xa * c[i] - xb * s[i]
            out[r, :, b] = xb * c[i] + xa * s[i]
    return out


def e4m3(x: np.ndarray) -> np.ndarray:
    """The nearest values of 4 exponent and 3 mantissa bits, ties to even, what is past 448 to 448; x in fp64.  Steps are 2^-9 up to
    2^-6 and an eighth of the power of two below from there on."""
    x = np.asarray(x, dtype=np.float64)
    size = np.where(np.isfinite(x), np.abs(x), 448.0)
    size = np.minimum(size, 448.0)
    step = np.exp2(np.floor(np.log2(np.maximum(size, 2.0 ** -6))) - 3)
    y = np.copysign(np.minimum(np.rint(size / step) * step, 448.0), x)
    return np.where(np.isnan(x), np.nan, y)


def least_exponent(x: np.ndarray) -> int:
    """The least e >= -117 with |x| <= 448 2^e for all finite x."""
    size = np.abs(x[np.isfinite(x)])
    top = float(size.max()) if size.size else 0.0
    e = LEAST
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


class Blocks:
    """Keys or values of one layer: codes as the numbers they stand for [pages, heads, tokens, d] and exponents [pages, heads, blocks], fp64
    and whole numbers, written token run by token run by the definition."""

    def __init__(self, n_pages: int, heads: int, page: int, d: int):
        self.code, self.e = np.zeros((n_pages, heads, page, d)), np.full((n_pages, heads, page // BLOCK), LEAST)
        self.page = page

    def put(self, pages, begin: int, x: np.ndarray):
        """Rows x [n, heads, d], positions begin .. begin + n - 1 of a sequence on `pages` (entries outside the cache: left out)."""
        n = len(x)
        at = begin
        while at < begin + n:
            stop = min((at // BLOCK + 1) * BLOCK, begin + n)
            if at >= 0 and at // self.page < len(pages) and 0 <= pages[at // self.page] < len(self.code):
                p, slot = pages[at // self.page], at % self.page
                b = slot // BLOCK
                for h in range(x.shape[1]):
                    new = x[at - begin:stop - begin, h].astype(np.float64)
                    e = least_exponent(new)
                    if slot % BLOCK:
                        old = int(np.clip(self.e[p, h, b], LEAST, MOST))
                        e = max(e, old)
                        if e > old:
                            lo = b * BLOCK
                            self.code[p, h, lo:slot] = e4m3(self.code[p, h, lo:slot] * 2.0 ** (old - e))
                    self.e[p, h, b] = e
                    y = e4m3(new * 2.0 ** -e)
                    if e == MOST:
                        y = np.where(np.abs(y) > 240, np.copysign(240.0, y), y)
                    self.code[p, h, slot:slot + len(new)] = y
            at = stop

    def values(self, pages, n: int) -> torch.Tensor:
        """[n, heads, d]: tokens 0 .. n - 1 of a sequence, 0 where a page is not there."""
        out = np.zeros((n, self.code.shape[1], self.code.shape[3]))
        for j in range(n):
            p = pages[j // self.page] if j // self.page < len(pages) else -1
            if 0 <= p < len(self.code):
                e = np.clip(self.e[p, :, j % self.page // BLOCK], LEAST, MOST)
                out[j] = self.code[p, :, j % self.page] * np.exp2(e.astype(np.float64))[:, None]
        return torch.from_numpy(out)
