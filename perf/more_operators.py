"""The work that the 4-bit operators are timed on.

A layer served in 4 bits is made of four calls, and each has its cases:

  * ``quantise``: activations become a matrix in microscaled 4-bit floating point
    (32 values share a power of two; ``vsk_mx4_quantise``), read back as values;
  * ``product``: activations, quantised within the call, times a weight matrix held
    in that format (``vsk_mx4_product``);
  * ``place``: the rows of a fused QKV projection: a norm and the rotation of each
    query and key head, queries out, K and V into the cache, in 16 or in 4 bits
    (``vsk_qkv_norm_rope``), and the new K and V read back;
  * ``attend``: attention over a cache held in 4 bits (``vsk_kv4_attend``), single
    tokens and prompt rows, over every key or through a window with sinks.

A case's sizes follow from the case alone; values come from the seed.
"""
from __future__ import annotations

import math
import random
import types

import numpy as np
import torch

own = False

BLOCK = 16
DEV = "cuda"
THETA = 500000.0
EPS = 1e-5
MAX_POS = 16384
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # magnitudes of a 4-bit value


# ------------------------------------------------------------------ cases
def _quant(name, rows, k, x="bf16"):
    return dict(name=name, kind="quantise", rows=rows, k=k, x=x)


def _product(name, rows, n, k, x="bf16", y="bf16", add=False):
    return dict(name=name, kind="product", rows=rows, n=n, k=k, x=x, y=y, add=add)


def _place(name, kv, group, hd, seqs, rows, past, bits, norm=True):
    return dict(name=name, kind="place", kv=kv, group=group, hd=hd, seqs=seqs, rows=rows, past=past, bits=bits, norm=norm)


def _attend(name, kv, group, hd, seqs, rows, lo, hi, window=0, sinks=0):
    return dict(name=name, kind="attend", kv=kv, group=group, hd=hd, seqs=seqs, rows=rows, lo=lo, hi=hi, window=window,
                sinks=sinks)


def listed():
    return [
        # a decode batch's normalised rows, as a projection takes them
        _quant("quantise_32", 32, 4096),
        # the gated activations of a prompt pass, one row more than whole tiles
        _quant("quantise_prompt", 2049, 14336),
        # one conversation's next token through the QKV projection
        _product("product_qkv_1", 1, 6144, 4096),
        # a decode batch through gate and up
        _product("product_gate_up_16", 16, 28672, 4096),
        # an odd batch through the down projection, added to the float32 residual stream
        _product("product_down_77", 77, 4096, 14336, y="fp32", add=True),
        # a prompt pass through gate and up
        _product("product_prompt", 2000, 28672, 4096),
        # a decode batch whose cache stays in 16 bits
        _place("place_decode_16", 8, 4, 128, 16, 1, 1000, 16),
        # fresh chunks of three prompts into a 4-bit cache
        _place("place_prompt_4bit", 8, 4, 128, 3, 611, 1205, 4),
        # the smallest attention: one short sequence of the one-layer test model
        _attend("attend_one", 4, 1, 64, 1, 1, 41, 41),
        # a full server's decode step
        _attend("attend_decode_64", 8, 4, 128, 64, 1, 2000, 12000),
        # two long documents: few rows, so the cache's length is what there is to split
        _attend("attend_long_2", 8, 4, 128, 2, 1, 15001, 16000),
        # later chunks of two prompts through a long window
        _attend("attend_prompt_window", 8, 4, 128, 2, 1000, 5500, 6003, window=4096, sinks=4),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_one(rng):
    kind = rng.choice(["quantise", "product", "product", "product", "place", "place", "attend", "attend", "attend"])
    hd = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 3, 4, 4, 6, 7, 8, 16])
    if kind == "quantise":
        c = _quant("", _log(rng, 1, 4096), _log(rng, 30, 16384), rng.choice(["bf16", "bf16", "fp32"]))
    elif kind == "product":
        c = _product("", _log(rng, 1, 4096), _log(rng, 16, 32768), _log(rng, 64, 16384),
                     rng.choice(["bf16", "bf16", "fp32", "mx4"]), rng.choice(["bf16", "fp32"]), rng.random() < 0.3)
    elif kind == "place":
        rows = rng.choice([1, 1, _log(rng, 2, 2000)])
        c = _place("", kv, group, hd, _log(rng, 1, 200) if rows == 1 else rng.randint(1, 5), rows,
                   rng.choice([0, _log(rng, 1, 12000)]), rng.choice([4, 4, 16]), rng.random() < 0.8)
    else:
        rows = rng.choice([1, 1, 1, _log(rng, 2, 1500)])
        hi = max(rows, _log(rng, 1, 16000))
        window = _log(rng, 1, 8192) if rng.random() < 0.4 else 0
        c = _attend("", kv, group, hd, _log(rng, 1, 150) if rows == 1 else rng.randint(1, 4), rows,
                    max(rows, int(hi * rng.uniform(0.2, 1.0))), hi, window,
                    rng.choice([0, 4, _log(rng, 1, 100)]) if window else 0)
    del c["name"]
    return c


def _cost(case):
    """Seconds that the case's work would take at a common pace of this card."""
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / (3e15 if case["kind"] == "product" else 8e14))


def draw(rng: random.Random):
    top = max(_cost(c) for c in listed())
    while True:
        c = _draw_one(rng)
        if _cost(c) <= top and (c["kind"] != "attend" or c["seqs"] * c["hi"] <= 800_000):
            return c


# ------------------------------------------------------------------ what a case's batch is
def _lens(case):
    """Cached tokens of each sequence, its new rows among them, in a mixed order."""
    n = case["seqs"]
    if case["kind"] == "place":
        return [case["past"] + case["rows"] + 3 * i for i in range(n)]
    lo, hi = case["lo"], case["hi"]
    x = [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]
    return x[::2] + x[1::2][::-1]


def _visible(p, window, sinks):
    """Keys that the row at index p sees."""
    if window == 0 or p + 1 <= window:
        return p + 1
    return window + min(sinks, p + 1 - window)


def _held(values):
    """Bytes of so many values in 4 bits, a byte more for each 32."""
    return values // 2 + values // 32


def work(case):
    kind = case["kind"]
    if kind == "quantise":
        n = case["rows"] * case["k"]
        return {"bytes": n * (4 if case["x"] == "fp32" else 2) + 2 * n, "flops": 4 * n}
    if kind == "product":
        rows, n, k = case["rows"], case["n"], case["k"]
        x = {"bf16": 2 * rows * k, "fp32": 4 * rows * k, "mx4": _held(rows * k)}[case["x"]]
        y = rows * n * (2 if case["y"] == "bf16" else 4)
        return {"bytes": x + _held(n * k) + y * (2 if case["add"] else 1), "flops": 2 * rows * n * k}
    kv, hd = case["kv"], case["hd"]
    heads = kv * case["group"]
    if kind == "place":
        rows = case["seqs"] * case["rows"]
        return {"bytes": rows * hd * 2 * (2 * heads + 4 * kv), "flops": 10 * rows * hd * (heads + kv)}
    nbytes, flops, rows, window, sinks = 0, 0, case["rows"], case["window"], case["sinks"]
    for total in _lens(case):
        lo = max(0, total - rows - window + 1) if window else 0
        keys = total - lo + min(sinks, lo)
        nbytes += 2 * _held(keys * kv * hd) + rows * heads * hd * 4
        flops += 4 * hd * heads * sum(_visible(p, window, sinks) for p in range(total - rows, total))
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------------ 4-bit values in plain operations
def _values(x):
    """x in microscaled 4 bits along its last axis: (values, exponents of 32 each).

    A block's exponent is floor(log2(largest magnitude)) - 2; its values are
    rounded to the grid of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to even steps, what
    is beyond 6 becomes 6."""
    n = x.shape[-1]
    b = torch.nn.functional.pad(x, (0, -n % 32)).unflatten(-1, (-1, 32))
    e = torch.clamp(torch.frexp(b.abs().amax(dim=-1)).exponent.to(torch.int32) - 3, min=-127)
    scale = torch.ldexp(torch.ones_like(b[..., 0]), e)[..., None]
    a = (b / scale).abs()
    step = torch.ldexp(torch.ones_like(a), torch.clamp(torch.frexp(a).exponent.to(torch.int32) - 2, -1, 1))
    v = torch.clamp(torch.round(a / step) * step, max=6.0)
    return (torch.copysign(v, b) * scale).flatten(-2)[..., :n], e


def _codes(x):
    """(codes, scales) of such a matrix as files hold it: two codes a byte, the
    first in its low half, and a biased exponent for each 32."""
    v, e = _values(x)
    n = x.shape[-1]
    b = torch.nn.functional.pad(v, (0, -n % 32)).unflatten(-1, (-1, 32))
    a = (b / torch.ldexp(torch.ones_like(b[..., 0]), e)[..., None])
    grid = torch.tensor(GRID, device=a.device)
    c = torch.bucketize(a.abs().float(), grid) + 8 * torch.signbit(a)
    c = c.flatten(-2)[..., :n + n % 2].to(torch.uint8)
    return c[..., 0::2] | c[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _held_values(codes, scales, n, dtype=torch.float32):
    """The values that codes and scales stand for, n of them in the last axis."""
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device, dtype=dtype)
    v = grid[torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).to(torch.int32)][..., :n]
    s = torch.ldexp(torch.ones(scales.shape, device=codes.device, dtype=dtype), scales.to(torch.int32) - 127)
    full = n // 32 * 32
    v[..., :full].unflatten(-1, (-1, 32)).mul_(s[..., :n // 32, None])
    if n % 32:
        v[..., full:].mul_(s[..., -1:])
    return v


# ------------------------------------------------------------------ inputs
def _gen(seed, at):
    return torch.Generator(device=DEV).manual_seed(seed * 1000003 + at)


def _activations(rows, k, seed, dtype):
    """Normalised rows: unit normal, one channel in 100 ten times as large."""
    x = torch.randn((rows, k), generator=_gen(seed, 1), device=DEV)
    x[:, torch.rand((k,), generator=_gen(seed, 2), device=DEV) < 0.01] *= 10.0
    return x.to(torch.bfloat16).to(DTYPE.get(dtype, torch.bfloat16))


def _weights(n, k, seed):
    """A weight matrix as a file holds it in 4 bits."""
    w = torch.randn((n, k), generator=_gen(seed, 3), device=DEV, dtype=torch.bfloat16)
    return _codes(w.float() * 0.02)


def _residual(case, seed):
    return torch.randn((case["rows"], case["n"]), generator=_gen(seed, 4), device=DEV).to(DTYPE[case["y"]])


def _layout(case):
    """Physical blocks of every sequence (a fixed permutation of a pool a little
    larger than needed) and the pool's size."""
    need = [(n + BLOCK - 1) // BLOCK for n in _lens(case)]
    pool = sum(need) + 3
    perm = np.random.default_rng(pool).permutation(pool).astype(np.int32)
    return np.split(perm[:sum(need)], np.cumsum(need)[:-1]), pool


def _slots(blocks, lo, hi):
    t = np.arange(lo, hi)
    return blocks[t // BLOCK].astype(np.int64) * BLOCK + t % BLOCK


def _kv(case, seed):
    """K and V of every cached token of every sequence, [tokens][kv][hd] bf16,
    sequence by sequence: unit normal, and one key in 50, with the first four of
    each sequence, along a direction that the queries share."""
    g = _gen(seed, 7)
    lens = _lens(case)
    total = sum(lens)
    K = torch.randn((total, case["kv"], case["hd"]), generator=g, device=DEV, dtype=torch.bfloat16)
    V = torch.randn((total, case["kv"], case["hd"]), generator=g, device=DEV, dtype=torch.bfloat16)
    heavy = torch.rand((total,), generator=g, device=DEV) < 0.02
    first = np.cumsum([0] + lens[:-1])
    heavy[torch.tensor([s + i for s, n in zip(first, lens) for i in range(min(4, n))], device=DEV)] = True
    K[..., 0] += heavy[:, None] * 6.0
    return K, V


def _q(case, seed):
    q = torch.randn((case["seqs"] * case["rows"], case["kv"] * case["group"], case["hd"]), generator=_gen(seed, 8),
                    device=DEV, dtype=torch.bfloat16)
    q[..., 0] += 4.0
    return q


def _qkv(case, seed):
    """Rows of a fused projection: queries, keys, values; and the gains of the norms."""
    heads = case["kv"] * (case["group"] + 2)
    x = torch.randn((case["seqs"] * case["rows"], heads * case["hd"]), generator=_gen(seed, 9), device=DEV,
                    dtype=torch.bfloat16)
    gains = 1.0 + 0.2 * torch.randn((2, case["hd"]), generator=_gen(seed, 10), device=DEV)
    return x * 1.7, gains.to(torch.bfloat16)


def _buffer(nbytes):
    """Device bytes whose address is a multiple of 256."""
    t = torch.empty(nbytes + 256, dtype=torch.uint8, device=DEV)
    return t, t.data_ptr() + (-t.data_ptr()) % 256


def prepare(case, seed):
    s = types.SimpleNamespace(case=case)
    if case["kind"] in ("quantise", "product"):
        _prepare_matrix(s, case, seed)
    else:
        _prepare_cache(s, case, seed)
    torch.cuda.synchronize()
    return s


def _prepare_matrix(s, case, seed):
    rows, k = case["rows"], case["k"]
    s.x = _activations(rows, k, seed, case["x"])
    if case["kind"] == "product":
        s.w = _weights(case["n"], k, seed)
        s.add = _residual(case, seed) if case["add"] else None
        if case["x"] == "mx4":
            s.x = _codes(s.x.float())
    if not own:
        return
    from paper_2609_37062_amd import vsk
    s.vsk, s.sp = vsk, torch.cuda.current_stream().cuda_stream
    if case["kind"] == "quantise":
        s.mx_t, s.mx = _buffer(vsk.mx4_bytes(rows, k))
        s.y = torch.empty((rows, k), dtype=torch.bfloat16, device=DEV)
        return

    def packed(m, n):
        t, at = _buffer(vsk.mx4_bytes(n, k))
        vsk.mx4_pack(m[0].data_ptr(), m[1].data_ptr(), n, k, at, s.sp)
        return t, at

    s.w_t, s.w_at = packed(s.w, case["n"])
    s.x_t, s.x_at = packed(s.x, rows) if case["x"] == "mx4" else (s.x, s.x.data_ptr())
    s.x_kind = {"bf16": vsk.BF16, "fp32": vsk.FP32, "mx4": vsk.MX4}[case["x"]]
    s.y_kind = {"bf16": vsk.BF16, "fp32": vsk.FP32}[case["y"]]
    s.y = torch.empty((rows, case["n"]), dtype=DTYPE[case["y"]], device=DEV)
    s.ws_bytes = vsk.mx4_product_bytes(rows, case["n"], k)
    s.ws_t, s.ws = _buffer(s.ws_bytes)


def _prepare_cache(s, case, seed):
    lens, rows = _lens(case), case["rows"]
    s.blocks, s.pool_blocks = _layout(case)
    if case["kind"] == "place":
        s.qkv, s.gains = _qkv(case, seed)
        s.pos = torch.tensor([p for n in lens for p in range(n - rows, n)], device=DEV)
        new = np.concatenate([_slots(b, n - rows, n) for b, n in zip(s.blocks, lens)])
        s.new_slots = torch.from_numpy(new.astype(np.int32)).to(DEV)
    else:
        K, V = _kv(case, seed)
        s.q = _q(case, seed)
    if own:
        _prepare_engine(s, case, lens)
        if case["kind"] == "attend":
            at = np.concatenate([_slots(b, 0, n) for b, n in zip(s.blocks, lens)]).astype(np.int32)
            at = torch.from_numpy(at).to(DEV)
            s.eng.kv4_write(0, at.data_ptr(), len(at), K.data_ptr(), V.data_ptr(), s.sp)
            torch.cuda.synchronize()
    elif case["kind"] == "attend":
        # the cache as a plain program keeps it: codes and scales by slot, and the
        # sequences' slots as one table (a short one's row ends in slot 0)
        slots = np.zeros((len(lens), max(lens)), np.int64)
        for i, (b, n) in enumerate(zip(s.blocks, lens)):
            slots[i, :n] = _slots(b, 0, n)
        s.slots = torch.from_numpy(slots).to(DEV)
        s.lens = torch.tensor(lens, device=DEV)
        at = s.slots[torch.arange(max(lens), device=DEV)[None, :] < s.lens[:, None]]
        s.cache = []
        for x in (K, V):
            codes, scales = _codes(x.float())
            c = torch.zeros((s.pool_blocks * BLOCK, *codes.shape[1:]), dtype=torch.uint8, device=DEV)
            e = torch.zeros((s.pool_blocks * BLOCK, *scales.shape[1:]), dtype=torch.uint8, device=DEV)
            c[at], e[at] = codes, scales
            s.cache.append((c, e))


def _prepare_engine(s, case, lens):
    """A handle whose sequences hold these blocks, and its uploaded batch."""
    from paper_2609_37062_amd import vsk
    m = types.SimpleNamespace(n_layers=1, hidden=1024, n_q_heads=case["kv"] * case["group"], n_kv_heads=case["kv"],
                              head_dim=case["hd"], ffn=1024, vocab=1024, max_pos=MAX_POS, rope_theta=THETA, rms_eps=EPS)
    s.sp = torch.cuda.current_stream().cuda_stream
    s.eng = e = vsk.Engine(m)
    if case["kind"] == "place" and case["bits"] == 16:
        s.pool_t, pool = _buffer(e.kv_pool_bytes(s.pool_blocks))
        e.kv_init(pool, s.pool_blocks)
    else:
        e.kv_init(None, s.pool_blocks)
        nbytes = e.kv4_pool_bytes(s.pool_blocks)
        s.pool_t, pool = _buffer(nbytes)
        e.kv4_init(pool, nbytes)
    for i, (b, n) in enumerate(zip(s.blocks, lens)):
        e.seq_create(i)
        e.seq_set_blocks(i, b, n)
    n_rows = case["seqs"] * case["rows"]
    e.batch_build(list(range(len(lens))), [case["rows"]] * len(lens))
    nbytes = e.batch_device_bytes()
    s.meta_t, meta = _buffer(nbytes)
    e.batch_upload(meta, nbytes, s.sp)
    if case["kind"] == "place":
        nbytes = e.rope_bytes()
        s.rope_t, rope = _buffer(nbytes)
        e.rope_bind(rope, nbytes, s.sp)
        s.q = torch.empty((n_rows, case["kv"] * case["group"], case["hd"]), dtype=torch.bfloat16, device=DEV)
        s.K = torch.empty((n_rows, case["kv"], case["hd"]), dtype=torch.bfloat16, device=DEV)
        s.V = torch.empty_like(s.K)
    else:
        s.o = torch.empty_like(s.q)
        cap = (n_rows, len(lens), max(lens))
        s.ws_bytes = e.workspace_bytes(*cap)
        s.ws_t, s.ws = _buffer(s.ws_bytes)
        e.workspace_init(s.ws, s.ws_bytes, *cap, s.sp)


# ------------------------------------------------------------------ one pass
def run(state):
    kind = state.case["kind"]
    if own:
        return {"quantise": _quantise_own, "product": _product_own, "place": _place_own, "attend": _attend_own}[kind](state)
    return {"quantise": _quantise_plain, "product": _product_plain, "place": _place_plain,
            "attend": _attend_plain}[kind](state)


def _quantise_own(s):
    c = s.case
    s.vsk.mx4_quantise(s.x.data_ptr(), s.vsk.FP32 if c["x"] == "fp32" else s.vsk.BF16, c["k"], c["rows"], c["k"], s.mx, s.sp)
    s.vsk.mx4_read(s.mx, c["rows"], c["k"], s.y.data_ptr(), s.vsk.BF16, c["k"], s.sp)
    return {"values": s.y}


def _quantise_plain(s):
    return {"values": _values(s.x.float())[0].to(torch.bfloat16)}


def _product_own(s):
    c = s.case
    s.vsk.mx4_product(s.x_at, s.x_kind, 0 if c["x"] == "mx4" else c["k"], s.w_at, c["rows"], c["n"], c["k"], s.y.data_ptr(),
                      s.y_kind, c["n"], s.ws, s.ws_bytes, add_ptr=s.add.data_ptr() if c["add"] else None, stream=s.sp)
    return {"y": s.y}


def _product_plain(s):
    c = s.case
    x = _held_values(*s.x, c["k"]) if c["x"] == "mx4" else _values(s.x.float())[0]
    y = torch.matmul(x, _held_values(*s.w, c["k"]).t())
    if c["add"]:
        y = y + s.add.float()
    return {"y": y.to(DTYPE[c["y"]])}


def _place_own(s):
    c, e = s.case, s.eng
    gq, gk = (s.gains[0].data_ptr(), s.gains[1].data_ptr()) if c["norm"] else (None, None)
    e.qkv_norm_rope(0, s.qkv.data_ptr(), s.qkv.shape[1], gq, gk, s.q.data_ptr(), c["bits"], s.sp)
    read = e.kv4_read if c["bits"] == 4 else e.kv_read
    read(0, s.new_slots.data_ptr(), len(s.new_slots), s.K.data_ptr(), s.V.data_ptr(), s.sp)
    return {"q": s.q, "K": s.K, "V": s.V}


def _place_plain(s):
    """Keys that go to 4 bits are taken in 64 bits until they are rounded: values
    lie next to the borders between two codes."""
    c = s.case
    kv, hd, heads = c["kv"], c["hd"], c["kv"] * c["group"]
    x = s.qkv.view(len(s.pos), heads + 2 * kv, hd)
    inv = torch.exp(torch.arange(hd // 2, device=DEV, dtype=torch.float64) * (-2.0 / hd * math.log(THETA)))
    angle = (s.pos.double()[:, None] * inv)[:, None, :]

    def turned(h, gain, dtype):
        h = h.to(dtype)
        if c["norm"]:
            h = h * torch.rsqrt((h * h).mean(dim=-1, keepdim=True) + EPS) * gain.to(dtype)
        a, b = h[..., :hd // 2], h[..., hd // 2:]
        cos, sin = torch.cos(angle).to(dtype), torch.sin(angle).to(dtype)
        return torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)

    q = turned(x[:, :heads], s.gains[0], torch.float32).to(torch.bfloat16)
    K = turned(x[:, heads:heads + kv], s.gains[1], torch.float64 if c["bits"] == 4 else torch.float32)
    V = x[:, heads + kv:]
    if c["bits"] == 4:
        K, V = _values(K)[0], _values(V.float())[0]
    return {"q": q, "K": K.to(torch.bfloat16), "V": V.to(torch.bfloat16)}


def _attend_own(s):
    c = s.case
    s.eng.kv4_attend(0, s.q.data_ptr(), s.o.data_ptr(), s.ws, s.ws_bytes, window=c["window"], sinks=c["sinks"], stream=s.sp)
    return {"o": s.o}


def _attend_plain(s):
    """Every sequence's cache gathered through the table and turned into float32,
    scores, mask, softmax and weighted sum, all sequences at once."""
    c = s.case
    n, rows, kv, group, hd = c["seqs"], c["rows"], c["kv"], c["group"], c["hd"]
    longest = s.slots.shape[1]
    K, V = (_held_values(codes[s.slots], scales[s.slots], hd) for codes, scales in s.cache)
    K = K.permute(0, 2, 3, 1).contiguous()  # [n][kv][hd][keys]
    V = V.permute(0, 2, 1, 3).contiguous()
    q = s.q.float().view(n, rows, kv, group, hd).permute(0, 2, 1, 3, 4).reshape(n, kv, rows * group, hd)
    sc = (torch.matmul(q, K) * (1.0 / math.sqrt(hd))).view(n, kv, rows, group, longest)
    p = (s.lens[:, None] - rows + torch.arange(rows, device=DEV))[:, :, None]
    t = torch.arange(longest, device=DEV)[None, None, :]
    seen = t <= p
    if c["window"]:
        seen &= (t > p - c["window"]) | (t < c["sinks"])
    sc = torch.where(seen[:, None, :, None, :], sc, -math.inf)
    e = torch.exp(sc - sc.amax(dim=-1, keepdim=True))
    w = (e / e.sum(dim=-1, keepdim=True)).view(n, kv, rows * group, longest)
    o = torch.matmul(w, V).view(n, kv, rows, group, hd).permute(0, 2, 1, 3, 4)
    return {"o": o.reshape(n * rows, kv * group, hd).to(torch.bfloat16)}


# ------------------------------------------------------------------ the definition, in 64 bits
def _nearest(x):
    """x rounded to 4-bit values by its distance to each of the grid's, 32 by 32."""
    x = x.double()
    out = torch.empty_like(x)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    middle = (grid[1:] + grid[:-1]) / 2
    for at in range(0, x.shape[-1], 32):
        b = x[..., at:at + 32]
        top = b.abs().amax(dim=-1, keepdim=True)
        # the largest power of two that is at most the largest magnitude, over 4
        p = torch.exp2(torch.floor(torch.log2(torch.clamp(top, min=2.0 ** -125))))
        p = torch.where(p > top, p / 2, torch.where(2 * p <= top, 2 * p, p)) / 4
        a = b.abs() / p
        low, high = torch.bucketize(a, middle), torch.bucketize(a, middle, right=True)
        i = torch.where(low == high, low, low + low % 2)  # between two: the even one
        out[..., at:at + 32] = torch.sign(b) * grid[i] * p
    return out


def _from_file(codes, scales, k):
    grid = torch.tensor(GRID, dtype=torch.float64, device=codes.device)
    c = torch.empty((*codes.shape[:-1], 2 * codes.shape[-1]), dtype=torch.int64, device=codes.device)
    c[..., 0::2], c[..., 1::2] = codes % 16, codes // 16
    v = grid[c % 8] * (1.0 - 2.0 * (c // 8))
    return v[..., :k] * torch.exp2(scales.double() - 127.0).repeat_interleave(32, dim=-1)[..., :k]


def exact(case, seed):
    kind = case["kind"]
    if kind == "quantise":
        return {"values": _nearest(_activations(case["rows"], case["k"], seed, case["x"]))}
    if kind == "product":
        x = _nearest(_activations(case["rows"], case["k"], seed, case["x"]))
        y = x @ _from_file(*_weights(case["n"], case["k"], seed), case["k"]).t().contiguous()
        return {"y": y + _residual(case, seed).double() if case["add"] else y}
    lens, rows, kv, group, hd = _lens(case), case["rows"], case["kv"], case["group"], case["hd"]
    if kind == "place":
        x, gains = _qkv(case, seed)
        x = x.double().view(-1, kv * (group + 2), hd)
        half = hd // 2
        pos = np.concatenate([np.arange(n - rows, n) for n in lens]).astype(np.float64)
        turn = torch.from_numpy(np.exp(1j * pos[:, None] * THETA ** (-np.arange(half) / half))).to(DEV)[:, None, :]
        parts = []
        for part, g in ((x[:, :kv * group], gains[0]), (x[:, kv * group:-kv], gains[1])):
            if case["norm"]:
                part = part / torch.sqrt(part.square().sum(dim=-1, keepdim=True) / hd + EPS) * g.double()
            z = torch.complex(part[..., :half], part[..., half:]) * turn
            parts.append(torch.cat((z.real, z.imag), dim=-1))
        q, K, V = *parts, x[:, -kv:]
        return {"q": q, "K": _nearest(K), "V": _nearest(V)} if case["bits"] == 4 else {"q": q, "K": K, "V": V}
    K, V = (_nearest(x) for x in _kv(case, seed))
    q = _q(case, seed)
    o = torch.empty(q.shape, dtype=torch.float64, device=DEV)
    k0 = 0
    for i, total in enumerate(lens):
        index = torch.arange(total, device=DEV)
        age = (total - rows + torch.arange(rows, device=DEV))[:, None] - index[None, :]
        hidden = age < 0
        if case["window"]:
            hidden |= (age >= case["window"]) & (index[None, :] >= case["sinks"])
        for h in range(kv * group):
            kh = K[k0:k0 + total, h // group].t().contiguous()
            z = q[i * rows:(i + 1) * rows, h].double() @ kh / hd ** 0.5
            o[i * rows:(i + 1) * rows, h] = torch.softmax(z.masked_fill(hidden, -math.inf), dim=1) @ V[k0:k0 + total, h // group]
        k0 += total
    return {"o": o}
