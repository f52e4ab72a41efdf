"""Paged 8-bit caches for the tests: made up, taken apart and appended to in 64 bits (by the layout that chunkflow.h describes)."""
import math

import numpy as np
import torch

DEV = "cuda:0"
#: half a step of e4m3 relative to a normal value, and of its subnormals (multiples of 2^-9)
E4M3_REL, E4M3_ABS = 2.0 ** -4, 2.0 ** -10
BF16_REL = 2.0 ** -8
ULP = 2.0 ** -24
E_LEAST = -100


def e4m3_values():
    v = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v[c] = (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) * (-1 if c & 128 else 1)
    v[0x7f] = v[0xff] = np.nan
    return v


E4M3 = e4m3_values()


class Cache:
    """Host copy: codes k [pages, heads, groups, hd / 16, 16, 16], v [pages, heads, groups, hd, 16], scales [pages, heads, groups, 2], table."""

    def __init__(self, rng, seqs, heads, hd, page, capacity, spare=2, fill="random"):
        groups, width = page // 16, max(1, -(-capacity // page))
        pages = seqs * width + spare
        self.page, self.heads, self.hd, self.pages = page, heads, hd, pages
        codes = lambda *s: (rng.integers(0, 128, s) % 127 + 128 * rng.integers(0, 2, s)).astype(np.uint8)       # noqa: E731   (no NaN)
        self.k, self.v = codes(pages, heads, groups, hd // 16, 16, 16), codes(pages, heads, groups, hd, 16)
        if fill == "small":                       # values up to 2, most of them ordinary ones
            for c in (self.k, self.v):
                c[:] = np.where((c & 127) >= 0x40, c & 0x3f | c & 128, c)
        self.scales = rng.integers(122, 130, (pages, heads, groups, 2)).astype(np.uint8)
        self.table = rng.permutation(pages)[:seqs * width].reshape(seqs, width).astype(np.int32)

    def device(self, B):
        t = [torch.from_numpy(x).to(DEV) for x in (self.k, self.v, self.scales, self.table)]
        return B.make_kv_cache(*t)

    def copy_back(self, cache):
        self.k, self.v, self.scales = (x.cpu().numpy() for x in cache.tensors[:3])

    def group(self, b, p):
        """(page, group) of position p of sequence b; None where there is none."""
        if p >= self.table.shape[1] * self.page:
            return None
        pg = int(self.table[b, p // self.page])
        return (pg, p % self.page // 16) if 0 <= pg < self.pages else None

    def held(self, b, n):
        """K, V [heads, n, hd] and which of the n tokens are there."""
        k, v, there = np.zeros((self.heads, n, self.hd)), np.zeros((self.heads, n, self.hd)), np.zeros(n, bool)
        for p in range(0, n, 16):
            at = self.group(b, p)
            if at is None:
                continue
            pg, g = at
            m = min(16, n - p)
            f = np.ldexp(1.0, self.scales[pg, :, g].astype(int) - 127)
            k[:, p:p + m] = (E4M3[self.k[pg, :, g]].transpose(0, 2, 1, 3).reshape(self.heads, 16, self.hd) * f[:, 0, None, None])[:, :m]
            v[:, p:p + m] = (E4M3[self.v[pg, :, g]].transpose(0, 2, 1) * f[:, 1, None, None])[:, :m]
            there[p:p + m] = True
        return k, v, there


def lens_t(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def attention(cache, q, cu, lens, causal, scale):
    """(o, tolerance) in 64 bits; NaN rows of o where no sequence has the row.
    Tolerance: weights rounded to bf16, whose sum is what divides (2^-8 (A + |o|), A the weighted mean of |v|), scores summed in fp32
    (hd + 8 roundings of sum |q k|), half a step of the result."""
    n_rows, heads, hd = q.shape
    times = heads // cache.heads
    o, tol = np.full(q.shape, np.nan), np.zeros(q.shape)
    for b, held in enumerate(lens):
        held = min(max(int(held), 0), cache.table.shape[1] * cache.page)
        k, v, there = cache.held(b, held)
        n = cu[b + 1] - cu[b]
        for i in range(n):
            row = cu[b] + i
            end = min(held, held - n + i + 1) if causal else held
            seen = there & (np.arange(held) < end)
            for h in range(heads):
                kk, vv = k[h // times][seen], v[h // times][seen]
                if not len(kk):
                    o[row, h] = 0
                    continue
                s = scale * (kk @ q[row, h])
                w = np.exp(s - s.max())
                w /= w.sum()
                o[row, h] = w @ vv
                mean = w @ np.abs(vv) + np.abs(o[row, h])
                off = (hd + 8) * ULP * scale * (np.abs(kk) @ np.abs(q[row, h])).max()
                tol[row, h] = mean * (1.01 * BF16_REL + 2 * off) + BF16_REL * np.abs(o[row, h]) + 1e-30
    return o, tol


def power(m):
    """The least power of two that holds m under 448."""
    if not m > 0:
        return E_LEAST
    e = math.frexp(m)[1] - 10
    while 448.0 * 2.0 ** e < m:
        e += 1
    return max(e, E_LEAST)
