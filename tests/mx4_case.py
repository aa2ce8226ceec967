"""Microscaled 4-bit values in 64 bits (numpy), from the format's definition, and an
engine whose cache is held in them."""
from __future__ import annotations

import numpy as np

from cache_case import BLOCK, Cache, bf16

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _blocks(x):
    n = x.shape[-1]
    pad = [(0, 0)] * (x.ndim - 1) + [(0, -n % 32)]
    return np.pad(np.asarray(x, np.float64), pad).reshape(*x.shape[:-1], -1, 32)


def exponents(x):
    """Biased exponents of the blocks of 32 along the last axis (255: not finite)."""
    top = np.abs(_blocks(x)).max(axis=-1)  # (NaN where one is)
    e = np.frexp(np.where(np.isfinite(top), top, 1.0))[1] - 1 - 2
    e = np.where(top == 0, -127, np.maximum(e, -127))
    return np.where(np.isfinite(top), e + 127, 255).astype(np.uint8)


def codes(x):
    """4-bit codes along the last axis: sign, and the nearest of the grid (ties: the
    even one)."""
    b, e = _blocks(x), exponents(x).astype(np.int64)
    bad = e == 255
    with np.errstate(invalid="ignore"):
        a = np.abs(np.ldexp(np.where(bad[..., None], 0.0, b), (127 - e)[..., None]))
    c = np.zeros(a.shape, np.uint8)
    for i in range(7):
        mid = (GRID[i] + GRID[i + 1]) / 2
        c[(a > mid) | ((a == mid) & (i % 2 == 1))] = i + 1
    c |= np.where(np.signbit(b) & ~bad[..., None], 8, 0).astype(np.uint8)
    return c.reshape(*x.shape[:-1], -1)[..., :x.shape[-1]]


def of_codes(c, e):
    """The values that codes and biased exponents stand for."""
    e = np.repeat(e.astype(np.int64), 32, axis=-1)[..., :c.shape[-1]]
    v = np.ldexp(GRID[c & 7] * np.where(c & 8, -1.0, 1.0), e - 127)
    return np.where(e == 255, np.nan, v)


def values(x):
    return of_codes(codes(x), exponents(x))


def in_file(c):
    """Two codes a byte, the first in its low half."""
    c = np.concatenate([c, np.zeros((*c.shape[:-1], c.shape[-1] % 2), np.uint8)], axis=-1)
    return np.ascontiguousarray(c[..., 0::2] | c[..., 1::2] << 4)


class Cache4(Cache):
    """A Cache in 4 bits: K and V are what the slots stand for."""

    def write(self, layer, seq, first=0):
        t = self.torch
        if not hasattr(self, "pool4"):
            n = self.eng.kv4_pool_bytes(self.n_blocks)
            self._pool4, at = self.buf(n, "cuda")
            self._pool4.fill_(-1)  # codes of -6, exponents that say NaN
            self.eng.kv4_init(at, n)
            self.pool4 = at
        n = len(self.K[layer][seq])
        s = t.from_numpy(self.slots(seq, n)[first:].astype(np.int32)).cuda()
        k, v = bf16(self.K[layer][seq][first:]).cuda(), bf16(self.V[layer][seq][first:]).cuda()
        self.eng.kv4_write(layer, s.data_ptr(), n - first, k.data_ptr(), v.data_ptr(), self.sp)
        t.cuda.synchronize()
        for x in (self.K, self.V):
            x[layer][seq][first:] = values(x[layer][seq][first:])

    def read(self, layer, seq):
        t = self.torch
        n, _ = self.eng.seq_info(seq)
        s = t.from_numpy(self.slots(seq, n).astype(np.int32)).cuda()
        k = t.zeros((n, self.kv, self.hd), dtype=t.bfloat16, device="cuda")
        v = t.zeros_like(k)
        self.eng.kv4_read(layer, s.data_ptr(), n, k.data_ptr(), v.data_ptr(), self.sp)
        t.cuda.synchronize()
        return k.float().cpu().numpy(), v.float().cpu().numpy()

    def attend(self, layer=0, window=0, sinks=0, stream=None):
        self.eng.kv4_attend(layer, self.qd.data_ptr(), self.o.data_ptr(), self.ws, self.ws_bytes, window=window,
                            sinks=sinks, stream=self.sp if stream is None else stream)


assert BLOCK == 16
