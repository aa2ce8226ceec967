"""Engines over a small drawn cache, and the bounded-cache operators in 64 bits.

The reference computes from the logical K, V and q of each sequence in float64
(numpy, CPU).  Bounds follow from the arithmetic of the kernels: products of
bf16 values summed in float32, exponents and weights in float32, a weight's
first 16 bits in the sum over V, one rounding to bf16.
"""
from __future__ import annotations

import types

import numpy as np

BLOCK = 16
U = 2.0 ** -24  # half a step of float32


def model(kv, group, hd, layers=1, max_pos=16384):
    return types.SimpleNamespace(n_layers=layers, hidden=256, n_q_heads=kv * group, n_kv_heads=kv, head_dim=hd, ffn=256,
                                 vocab=256, max_pos=max_pos, rope_theta=500000.0, rms_eps=1e-5)


def bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16)


class Cache:
    """One engine whose sequences 0, 1, .. hold drawn K, V at permuted blocks."""

    def __init__(self, kv, group, hd, lens, layers=1, seed=0, spare=64, tables=None, max_pos=16384, scale=1.0):
        import torch
        from paper_2609_37062_amd import vsk
        from paper_2609_37062_amd.runner import _dev_buffer
        self.torch, self.vsk, self.buf = torch, vsk, _dev_buffer
        self.kv, self.group, self.hd, self.layers, self.lens = kv, group, hd, layers, list(lens)
        rng = np.random.default_rng(seed)
        self.rng = rng
        self.eng = vsk.Engine(model(kv, group, hd, layers, max_pos))
        need = [(n + BLOCK - 1) // BLOCK for n in lens]
        self.n_blocks = sum(need) + spare
        perm = rng.permutation(self.n_blocks).astype(np.int32)
        self.pool = torch.full((self.eng.kv_pool_bytes(self.n_blocks) // 2,), -1, dtype=torch.int16, device="cuda")
        self.eng.kv_init(self.pool.data_ptr(), self.n_blocks)
        self.K, self.V = [], []  # [layer][sequence] float32 arrays holding bf16 values, [len][kv][hd]
        at, blocks = 0, []
        for i, n in enumerate(need):
            blocks.append(perm[at:at + n] if tables is None or tables[i] is None else np.asarray(tables[i], np.int32))
            at += n
            self.eng.seq_create(i)
            self.eng.seq_set_blocks(i, blocks[i], lens[i])
        self.blocks = blocks
        for l in range(layers):
            self.K.append([bf16(scale * rng.standard_normal((n, kv, hd))).float().numpy() for n in lens])
            self.V.append([bf16(rng.standard_normal((n, kv, hd))).float().numpy() for n in lens])
        self.sp = torch.cuda.current_stream().cuda_stream
        for l in range(layers):
            for i in range(len(lens)):
                self.write(l, i)

    def slots(self, seq, n):
        t = np.arange(n)
        _, table = self.eng.seq_info(seq)
        return np.asarray(table, np.int64)[t // BLOCK] * BLOCK + t % BLOCK

    def write(self, layer, seq, first=0):
        """(Again) the K, V of a sequence from its logical values."""
        t = self.torch
        n = len(self.K[layer][seq])
        s = t.from_numpy(self.slots(seq, n)[first:].astype(np.int32)).cuda()
        k = bf16(self.K[layer][seq][first:]).cuda()
        v = bf16(self.V[layer][seq][first:]).cuda()
        self.eng.kv_write(layer, s.data_ptr(), n - first, k.data_ptr(), v.data_ptr(), self.sp)
        t.cuda.synchronize()

    def read(self, layer, seq):
        t = self.torch
        n, _ = self.eng.seq_info(seq)
        s = t.from_numpy(self.slots(seq, n).astype(np.int32)).cuda()
        k = t.empty((n, self.kv, self.hd), dtype=t.bfloat16, device="cuda")
        v = t.empty_like(k)
        self.eng.kv_read(layer, s.data_ptr(), n, k.data_ptr(), v.data_ptr(), self.sp)
        t.cuda.synchronize()
        return k.float().cpu().numpy(), v.float().cpu().numpy()

    def batch(self, seqs, q_lens):
        t = self.torch
        self.seqs, self.q_lens = list(seqs), list(q_lens)
        self.eng.batch_build(seqs, q_lens)
        n = self.eng.batch_device_bytes()
        self._meta, meta = self.buf(n, "cuda")
        self.eng.batch_upload(meta, n, self.sp)
        cap = (sum(q_lens), len(seqs), max(self.eng.seq_info(s)[0] for s in seqs))
        self.ws_bytes = self.eng.workspace_bytes(*cap)
        self._ws, self.ws = self.buf(self.ws_bytes, "cuda")
        self.eng.workspace_init(self.ws, self.ws_bytes, *cap, self.sp)
        rows = sum(q_lens)
        self.q = bf16(self.rng.standard_normal((rows, self.kv * self.group, self.hd)))
        self.qd = self.q.cuda()
        self.o = t.full((rows + 1, self.kv * self.group, self.hd), -7.0, dtype=t.bfloat16, device="cuda")
        t.cuda.synchronize()

    def attend(self, layer=0, window=0, sinks=0, mass=None, add=False, stream=None):
        self.eng.attend(layer, self.qd.data_ptr(), self.o.data_ptr(), self.ws, self.ws_bytes, window=window, sinks=sinks,
                        mass_ptr=None if mass is None else mass.data_ptr(),
                        mass_stride=0 if mass is None else mass.shape[1], mass_add=add,
                        stream=self.sp if stream is None else stream)

    def out(self):
        self.torch.cuda.synchronize()
        o = self.o.float().cpu().numpy()
        assert (o[-1] == -7.0).all(), "the row behind the last one was written"
        return o[:-1].astype(np.float64)

    def close(self):
        self.torch.cuda.synchronize()
        self.eng.close()


def visible(p, n, window, sinks):
    """Which of n keys the row at index p sees."""
    t = np.arange(n)
    m = t <= p
    if window:
        m &= (t > p - window) | (t < sinks)
    return m


def attend_ref(q, K, V, first, window, sinks):
    """Rows q [rows][heads][hd] at indexes first, first + 1, ..: the output, its
    bound, the weight per key over rows and heads, and its bound."""
    q, K, V = (np.asarray(x, np.float64) for x in (q, K, V))
    rows, heads, hd = q.shape
    n, kv = K.shape[:2]
    G = heads // kv
    o, ob = np.zeros(q.shape), np.zeros(q.shape)
    mass, mb = np.zeros(n), np.zeros(n)
    for r in range(rows):
        see = np.flatnonzero(visible(first + r, n, window, sinks))
        for h in range(heads):
            k, v = K[see, h // G], V[see, h // G]
            s = k @ q[r, h] / np.sqrt(hd)
            w = np.exp(s - s.max())
            w /= w.sum()
            # a score is off by at most (hd + 2) roundings of its largest partial
            # sum, an exponent by two roundings of the scaled score more, and the
            # normalised weight by twice that and the roundings of its sum
            ds = (hd + 2) * U * (np.abs(k) @ np.abs(q[r, h])).max() / np.sqrt(hd) + 4 * U * (np.abs(s).max() + 1)
            dw = 2 * ds + (len(see) / 32 + 64) * U
            o[r, h] = w @ v
            # (2^-16: a weight's bits behind the sixteenth; 2^-8 of the value: the bf16 output)
            ob[r, h] = (dw + 2.0 ** -16 + (len(see) / 32 + 64) * U) * (w @ np.abs(v)) + 2.0 ** -8 * np.abs(o[r, h])
            mass[see] += w
            mb[see] += w * dw
    return o, ob * (1 + 2.0 ** -7) + 1e-30, mass, mb + mass * (rows * heads / 16 + 80) * U + 1e-30


def check(c, window=0, sinks=0, layer=0, mass=None, base=None):
    """The outputs of the last attend call against the reference; returns it."""
    got, r0, out = c.out(), 0, []
    m = None if mass is None else mass.cpu().numpy().astype(np.float64)
    for i, (s, ql) in enumerate(zip(c.seqs, c.q_lens)):
        n = len(c.K[layer][s])
        o, ob, ms, mb = attend_ref(c.q[r0:r0 + ql].float().numpy(), c.K[layer][s], c.V[layer][s], n - ql, window, sinks)
        err = np.abs(got[r0:r0 + ql] - o)
        assert (err <= ob).all(), (i, n, ql, float(np.nanmax(err / ob)), np.argwhere(~(err <= ob))[:4].tolist())
        if m is not None:
            want = ms + (0 if base is None else base[i, :n])
            e = np.abs(m[i, :n] - want)
            b = mb + (0 if base is None else 2 * U * np.abs(want))
            assert (e <= b).all(), (i, n, ql, float(np.nanmax(e / b)))
        out.append((o, ms))
        r0 += ql
    return out
