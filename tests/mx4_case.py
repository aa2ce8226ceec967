"""Microscaled 4-bit values in 64 bits (numpy), from the format's definition, and an
engine whose cache is held in them."""
from __future__ import annotations

import numpy as np

from cache_case import BLOCK, Cache, attend_ref, bf16

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


def check_rows(c, window=0, sinks=0, layer=0):
    """As check, of prompt rows.  Beyond what that counts, a weight w_i, taken with 11
    bits, is off by at most 2^-11 w_i (half a step of fp16), or by half of fp16's
    smallest step where it is below 2^-14.  Weights go in as 2^7 times their ratio to a
    maximum that the row's largest ratio exceeds by 1 to 2^8, and their sum is at least
    2^7; so the second is at most 2^-25 / 2^7 of the sum, a key."""
    got, r0 = c.out(), 0
    for i, (s, ql) in enumerate(zip(c.seqs, c.q_lens)):
        q, K, V = c.q[r0:r0 + ql].float().numpy(), c.K[layer][s], c.V[layer][s]
        n = len(K)
        o, ob, _, _ = attend_ref(q, K, V, n - ql, window, sinks)
        oa, _, _, _ = attend_ref(q, K, np.abs(V), n - ql, window, sinks)
        # (a key that a row does not see gives it nothing: the largest of those that it may)
        see = n if window == 0 else min(n, window + sinks)
        top = np.stack([np.abs(V[np.r_[:min(t + 1, sinks), max(0, t + 1 - window) if window else 0:t + 1]]).max(axis=0) for t in range(n - ql, n)])
        top = np.repeat(top, c.group, axis=1).reshape(o.shape)
        b = ob + 2.0 ** -11 * oa.reshape(o.shape) + see * 2.0 ** -32 * top
        err = np.abs(got[r0:r0 + ql] - o)
        assert (err <= b).all(), (i, n, ql, float(np.nanmax(err / b)), np.argwhere(~(err <= b))[:4].tolist())
        r0 += ql


def turned(x, pos, gain, theta, eps):
    """[rows][heads][hd] in 64 bits; also the magnitudes of the terms."""
    hd = x.shape[-1]
    if gain is not None:
        x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * gain
    a = (pos[:, None] * theta ** (-2.0 * np.arange(hd // 2) / hd))[:, None, :]
    lo, hi = x[..., :hd // 2], x[..., hd // 2:]
    y = np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], axis=-1)
    m = np.concatenate([np.abs(lo * np.cos(a)) + np.abs(hi * np.sin(a)), np.abs(hi * np.cos(a)) + np.abs(lo * np.sin(a))], axis=-1)
    return y, m


assert BLOCK == 16
