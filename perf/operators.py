"""The work that the bounded-cache operators are timed on.

Three calls keep a long-running sequence's cache bounded, and each has its cases:

  * ``attend``: attention of the batch's rows over the paged cache
    (``vsk_attend``), single tokens and prompt rows, over every key or over a
    sliding window and a few first keys that stay visible;
  * the same call with ``mass``: it also returns, per cached token, the
    attention weight that the rows gave it;
  * ``evict``: a sequence keeps its most attended tokens (``vsk_kv_evict``) and
    goes on with a shorter cache.

A case's lengths follow from the case alone; values come from the seed.  K, V
and q are drawn so that attention is neither flat nor one-hot: unit normal
scores, and a few keys of each sequence (its first ones among them) that many
queries agree with.
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


# ------------------------------------------------------------------ cases
def _attend(name, kv, group, hd, decodes=0, lo=0, hi=0, prompts=0, plen=0, past=0, window=0, sinks=0, mass=False):
    return dict(name=name, kind="attend", kv=kv, group=group, hd=hd, decodes=decodes, lo=lo, hi=hi, prompts=prompts,
                plen=plen, past=past, window=window, sinks=sinks, mass=mass)


def _evict(name, kv, hd, layers, seqs, lo, hi, keep, sinks, recent):
    return dict(name=name, kind="evict", kv=kv, hd=hd, layers=layers, seqs=seqs, lo=lo, hi=hi, keep=keep, sinks=sinks,
                recent=recent)


def listed():
    return [
        # the smallest call: one short sequence of the one-layer test model; a launch is all there is
        _attend("attend_one", 4, 1, 64, decodes=1, lo=41, hi=41),
        # a small chat batch, every key visible
        _attend("attend_decode_16", 8, 4, 128, decodes=16, lo=512, hi=1024),
        # two long documents: few rows, so the cache's length is what there is to split
        _attend("attend_long_2", 8, 4, 128, decodes=2, lo=15001, hi=16000),
        # a full server whose layers see a window and four first tokens of long sequences
        _attend("attend_window_128", 8, 4, 128, decodes=128, lo=700, hi=16000, window=1024, sinks=4),
        # a full server on layers without a window
        _attend("attend_decode_64", 8, 3, 128, decodes=64, lo=2000, hi=12000),
        # fresh prompts of an odd length through a short window
        _attend("attend_prompt_window", 8, 3, 128, prompts=4, plen=1037, window=256, sinks=4),
        # a later chunk of a long document beside decoding sequences, a long window
        _attend("attend_chunk_mixed", 8, 4, 128, decodes=7, lo=300, hi=3000, prompts=1, plen=1000, past=7003,
                window=4096, sinks=16),
        # a decode step that counts what each cached token is worth
        _attend("mass_decode_32", 8, 4, 128, decodes=32, lo=1000, hi=4000, mass=True),
        # a prompt whose rows leave their weights, so that its cache can be cut behind it
        _attend("mass_prompt_777", 8, 4, 128, prompts=1, plen=777, past=2300, mass=True),
        # one short sequence of the test model is cut to half
        _evict("evict_one", 4, 64, 1, 1, 201, 201, 96, 4, 32),
        # eight conversations are cut to a budget of 1,000 tokens, a few layers
        _evict("evict_8", 8, 128, 8, 8, 3000, 5001, 1000, 4, 256),
        # long documents are cut to a quarter, half a model's layers
        _evict("evict_long_3", 8, 128, 16, 3, 15001, 16000, 4096, 16, 1024),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_one(rng):
    kind = rng.choice(["decode", "decode", "decode", "prompt", "prompt", "mixed", "evict", "evict"])
    hd = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8, 8])
    if kind == "evict":
        seqs = _log(rng, 1, 24)
        hi = _log(rng, 24, 16000)
        lo = max(2, int(hi * rng.uniform(0.3, 1.0)))
        keep = max(1, int(lo * rng.uniform(0.1, 1.0)))
        sinks = rng.randint(0, min(64, keep))
        recent = rng.randint(0, keep - sinks)
        c = _evict("", kv, hd, _log(rng, 1, 16), seqs, lo, hi, keep, sinks, recent)
    else:
        group = rng.choice([1, 2, 3, 4, 4, 6, 7, 8, 16])
        window, sinks = 0, 0
        if rng.random() < 0.6:
            window = _log(rng, 1, 8192)
            sinks = rng.choice([0, 4, _log(rng, 1, 100)])
        kw = {}
        if kind in ("decode", "mixed"):
            hi = _log(rng, 1, 16000)
            kw.update(decodes=_log(rng, 1, 200), lo=max(1, int(hi * rng.uniform(0.05, 1.0))), hi=hi)
        if kind in ("prompt", "mixed"):
            plen = _log(rng, 2, 2000)
            kw.update(prompts=rng.randint(1, 5), plen=plen, past=rng.choice([0, _log(rng, 1, 16000 - plen)]))
        c = _attend("", kv, group, hd, window=window, sinks=sinks, mass=rng.random() < 0.35, **kw)
    del c["name"]
    return c


def _cost(case):
    """Seconds that the case's work would take at a common pace of this card."""
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


def draw(rng: random.Random):
    top = max(_cost(c) for c in listed())
    while True:
        c = _draw_one(rng)
        if _cost(c) <= top and _tokens(c) <= 700_000:
            return c


# ------------------------------------------------------------------ what a case's batch is
def _spread(n, lo, hi):
    """n lengths from lo to hi, evenly spread, in a mixed order."""
    if n == 1:
        return [hi]
    x = [lo + (hi - lo) * i // (n - 1) for i in range(n)]
    return [x[(i * 7 + 3) % n] if n % 7 else x[(i * 5 + 2) % n] if n % 5 else x[n - 1 - i] for i in range(n)]


def _seqs(case):
    """(cached tokens with the new rows, new rows) of each sequence: prompts, then decodes."""
    if case["kind"] == "evict":
        return [(n, 0) for n in _spread(case["seqs"], case["lo"], case["hi"])]
    out = [(case["past"] + case["plen"], case["plen"])] * case["prompts"]
    if case["decodes"]:
        out += [(n, 1) for n in _spread(case["decodes"], case["lo"], case["hi"])]
    return out


def _tokens(case):
    return sum(n for n, _ in _seqs(case)) * (case["layers"] if case["kind"] == "evict" else 1)


def _visible(p, window, sinks):
    """Keys that the row at index p sees."""
    if window == 0 or p + 1 <= window:
        return p + 1
    return window + min(sinks, p + 1 - window)


def work(case):
    kv, hd = case["kv"], case["hd"]
    token = 2 * kv * hd * 2  # K and V of one token, bf16
    if case["kind"] == "evict":
        keep, n = case["keep"], case["seqs"]
        total = sum(t for t, _ in _seqs(case))
        moved = 2 * case["layers"] * keep * n * token  # read and written
        return {"bytes": moved + 4 * total + 12 * keep * n, "flops": total}
    heads = kv * case["group"]
    nbytes, flops = 0, 0
    for total, rows in _seqs(case):
        lo = max(0, total - rows - case["window"] + 1) if case["window"] else 0
        keys = total - lo + min(case["sinks"], lo)
        nbytes += keys * token + rows * heads * hd * 4 + (4 * total if case["mass"] else 0)
        flops += 4 * hd * heads * sum(_visible(p, case["window"], case["sinks"]) for p in range(total - rows, total))
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------------ inputs
def _layout(case):
    """Physical blocks of every sequence (a fixed permutation of a pool a little
    larger than needed) and the pool's size."""
    need = [(n + BLOCK - 1) // BLOCK for n, _ in _seqs(case)]
    spare = case["seqs"] * ((case["keep"] + BLOCK - 1) // BLOCK) if case["kind"] == "evict" else 3
    pool = sum(need) + spare
    perm = np.random.default_rng(pool).permutation(pool).astype(np.int32)
    out, at = [], 0
    for n in need:
        out.append(perm[at:at + n])
        at += n
    return out, pool


def _slots(blocks, n):
    t = np.arange(n)
    return blocks[t // BLOCK].astype(np.int64) * BLOCK + t % BLOCK


def _kv(case, seed, layer):
    """K and V of every cached token of every sequence, [tokens][kv][hd] bf16,
    sequence by sequence: unit normal, and one key in 50, with the first four of
    each sequence, along a direction that the queries share."""
    g = torch.Generator(device=DEV).manual_seed(seed * 1000003 + layer * 101 + 7)
    lens = [n for n, _ in _seqs(case)]
    total, kv, hd = sum(lens), case["kv"], case["hd"]
    K = torch.randn((total, kv, hd), generator=g, device=DEV, dtype=torch.bfloat16)
    V = torch.randn((total, kv, hd), generator=g, device=DEV, dtype=torch.bfloat16)
    heavy = torch.rand((total,), generator=g, device=DEV) < 0.02
    heavy[torch.tensor([s + i for s, n in zip(np.cumsum([0] + lens[:-1]), lens) for i in range(min(4, n))],
                       device=DEV)] = True
    K[..., 0] += heavy[:, None] * 6.0
    return K, V


def _q(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 1000003 + 3)
    rows = sum(r for _, r in _seqs(case))
    q = torch.randn((rows, case["kv"] * case["group"], case["hd"]), generator=g, device=DEV, dtype=torch.bfloat16)
    q[..., 0] += 4.0
    return q


def _mass(case, seed):
    """Accumulated weights as a server has them: heavy-tailed, many tokens never
    attended (0), some equal ones; [sequences][longest]."""
    g = torch.Generator(device=DEV).manual_seed(seed * 1000003 + 5)
    lens = [n for n, _ in _seqs(case)]
    x = torch.rand((len(lens), max(lens)), generator=g, device=DEV)
    m = torch.exp(4.0 * torch.randn(x.shape, generator=g, device=DEV))
    m[x < 0.3] = 0.0
    return torch.where(x > 0.9, torch.round(m), m)


def prepare(case, seed):
    s = types.SimpleNamespace(case=case)
    seqs = _seqs(case)
    lens = [n for n, _ in seqs]
    blocks, pool = _layout(case)
    slots = np.concatenate([_slots(b, n) for b, n in zip(blocks, lens)])
    s.slots = torch.from_numpy(slots).to(DEV)
    s.layers = case["layers"] if case["kind"] == "evict" else 1
    if case["kind"] == "evict":
        s.mass = _mass(case, seed)
    else:
        s.q = _q(case, seed)
        s.o = torch.empty_like(s.q)
        if case["mass"]:
            s.mass = torch.zeros((len(seqs), max(lens)), device=DEV)
    if not own:
        # the cache as a plain program keeps it: [layer][slot][kv][hd]
        s.K = torch.zeros((s.layers, pool * BLOCK, case["kv"], case["hd"]), dtype=torch.bfloat16, device=DEV)
        s.V = torch.zeros_like(s.K)
        for l in range(s.layers):
            s.K[l][s.slots], s.V[l][s.slots] = _kv(case, seed, l)
        s.seq_slots = list(torch.split(s.slots, lens))
        return s
    _prepare_own(s, case, seed, blocks, pool)
    return s


def _buffer(nbytes):
    """Device bytes whose address is a multiple of 256."""
    t = torch.empty(nbytes + 256, dtype=torch.uint8, device=DEV)
    return t, t.data_ptr() + (-t.data_ptr()) % 256


def _prepare_own(s, case, seed, blocks, pool):
    """A handle whose cache holds the same tokens at the same blocks."""
    from paper_2609_37062_amd import vsk
    seqs = _seqs(case)
    lens = [n for n, _ in seqs]
    group = case.get("group", 1)
    m = types.SimpleNamespace(n_layers=s.layers, hidden=1024, n_q_heads=case["kv"] * group, n_kv_heads=case["kv"],
                              head_dim=case["hd"], ffn=1024, vocab=1024, max_pos=16384, rope_theta=500000.0,
                              rms_eps=1e-5)
    s.sp = torch.cuda.current_stream().cuda_stream
    s.eng = e = vsk.Engine(m)
    s.pool = torch.zeros(e.kv_pool_bytes(pool) // 2, dtype=torch.int16, device=DEV)
    e.kv_init(s.pool.data_ptr(), pool)
    for i, (b, n) in enumerate(zip(blocks, lens)):
        e.seq_create(i)
        e.seq_set_blocks(i, b, n)
    slots32 = s.slots.to(torch.int32)
    for l in range(s.layers):
        K, V = _kv(case, seed, l)
        e.kv_write(l, slots32.data_ptr(), len(slots32), K.data_ptr(), V.data_ptr(), s.sp)
    if case["kind"] == "evict":
        n, keep = case["seqs"], case["keep"]
        s.src, s.dst, s.keep = list(range(n)), list(range(n, 2 * n)), [keep] * n
        s.meta_bytes = e.kv_evict_bytes(s.src, s.keep)
        s.meta_t, s.meta = _buffer(s.meta_bytes)
        s.kept = torch.empty((n, keep), dtype=torch.int32, device=DEV)
        s.new_slots = torch.empty((n, keep), dtype=torch.int32, device=DEV)
        s.mass_out = torch.empty((n, keep), device=DEV)
        s.outK = torch.empty((s.layers, n, keep, case["kv"], case["hd"]), dtype=torch.bfloat16, device=DEV)
        s.outV = torch.empty_like(s.outK)
    else:
        e.batch_build(list(range(len(seqs))), [r for _, r in seqs])
        s.meta_bytes = e.batch_device_bytes()
        s.meta_t, s.meta = _buffer(s.meta_bytes)
        e.batch_upload(s.meta, s.meta_bytes, s.sp)
        cap = (sum(r for _, r in seqs), len(seqs), max(lens))
        s.ws_bytes = e.workspace_bytes(*cap)
        s.ws_t, s.ws = _buffer(s.ws_bytes)
        e.workspace_init(s.ws, s.ws_bytes, *cap, s.sp)
    torch.cuda.synchronize()


# ------------------------------------------------------------------ one pass
def run(state):
    if state.case["kind"] == "evict":
        return _evict_own(state) if own else _evict_plain(state)
    return _attend_own(state) if own else _attend_plain(state)


def _attend_own(s):
    c = s.case
    s.eng.attend(0, s.q.data_ptr(), s.o.data_ptr(), s.ws, s.ws_bytes, window=c["window"], sinks=c["sinks"],
                 mass_ptr=s.mass.data_ptr() if c["mass"] else None, mass_stride=s.mass.shape[1] if c["mass"] else 0,
                 stream=s.sp)
    return {"o": s.o, "mass": s.mass} if c["mass"] else {"o": s.o}


def _attend_plain(s):
    """Per sequence: its keys gathered through the block table, scores, mask,
    softmax and weighted sum in float32."""
    c = s.case
    kv, group, hd, window, sinks = c["kv"], c["group"], c["hd"], c["window"], c["sinks"]
    o = torch.empty_like(s.q)
    mass = torch.zeros_like(s.mass) if c["mass"] else None
    at = 0
    for i, (total, rows) in enumerate(_seqs(c)):
        K = s.K[0][s.seq_slots[i]].float().permute(1, 2, 0).contiguous()  # [kv][hd][keys]
        V = s.V[0][s.seq_slots[i]].float().permute(1, 0, 2).contiguous()  # [kv][keys][hd]
        q = s.q[at:at + rows].float().view(rows, kv, group * hd).permute(1, 0, 2).reshape(kv, rows * group, hd)
        sc = torch.matmul(q, K) * (1.0 / math.sqrt(hd))
        if rows > 1 or window:
            p = torch.arange(total - rows, total, device=DEV)[:, None]
            t = torch.arange(total, device=DEV)[None, :]
            seen = t <= p
            if window:
                seen &= (t > p - window) | (t < sinks)
            seen = seen[:, None, :].expand(rows, group, total).reshape(rows * group, total)
            sc = torch.where(seen, sc, -math.inf)
        e = torch.exp(sc - sc.amax(dim=-1, keepdim=True))
        w = e / e.sum(dim=-1, keepdim=True)
        r = torch.matmul(w, V).view(kv, rows, group, hd).permute(1, 0, 2, 3).reshape(rows, kv * group, hd)
        o[at:at + rows] = r.to(o.dtype)
        if c["mass"]:
            mass[i, :total] = w.sum(dim=(0, 1))
        at += rows
    return {"o": o, "mass": mass} if c["mass"] else {"o": o}


def _evict_own(s):
    """The sequences move to shorter ones (released again afterwards, so that
    the call can be repeated), and their new cache is read."""
    c, e = s.case, s.eng
    n, keep = c["seqs"], c["keep"]
    for d in s.dst:
        e.seq_create(d)
    e.kv_evict(s.dst, s.src, s.keep, c["sinks"], c["recent"], s.mass.data_ptr(), s.mass.shape[1], s.meta, s.meta_bytes,
               mass_out_ptr=s.mass_out.data_ptr(), kept_ptr=s.kept.data_ptr(), slots_ptr=s.new_slots.data_ptr(),
               out_stride=keep, stream=s.sp)
    for l in range(s.layers):
        e.kv_read(l, s.new_slots.data_ptr(), n * keep, s.outK[l].data_ptr(), s.outV[l].data_ptr(), s.sp)
    for d in s.dst:
        e.seq_release(d)
    return {"kept": s.kept, "mass": s.mass_out, "K": s.outK, "V": s.outV}


def _evict_plain(s):
    """Per sequence: a stable descending sort of the middle's weights (equal
    ones in index order), the kept indexes in order, and their K, V and weights."""
    c = s.case
    n, keep, sinks, recent = c["seqs"], c["keep"], c["sinks"], c["recent"]
    kept, mass, slots = [], [], []
    for i, (total, _) in enumerate(_seqs(c)):
        mid = s.mass[i, sinks:total - recent]
        best = torch.sort(mid, descending=True, stable=True).indices[:keep - sinks - recent] + sinks
        idx = torch.cat([torch.arange(sinks, device=DEV), torch.sort(best).values,
                         torch.arange(total - recent, total, device=DEV)])
        kept.append(idx)
        mass.append(s.mass[i][idx])
        slots.append(s.seq_slots[i][idx])
    sl = torch.cat(slots)
    shape = (s.layers, n, keep, c["kv"], c["hd"])
    return {"kept": torch.stack(kept).to(torch.int32), "mass": torch.stack(mass), "K": s.K[:, sl].view(shape),
            "V": s.V[:, sl].view(shape)}


# ------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    seqs = _seqs(case)
    lens = [n for n, _ in seqs]
    if case["kind"] == "evict":
        # order by (weight descending, index ascending), on the host
        m = _mass(case, seed).cpu().numpy()
        n, keep, sinks, recent = case["seqs"], case["keep"], case["sinks"], case["recent"]
        kept = np.empty((n, keep), np.int32)
        for i, total in enumerate(lens):
            mid = np.arange(sinks, total - recent)
            order = mid[np.lexsort((mid, -m[i, mid].astype(np.float64)))]
            kept[i] = np.sort(np.concatenate([np.arange(sinks), order[:keep - sinks - recent],
                                              np.arange(total - recent, total)]))
        first = np.cumsum([0] + lens[:-1])
        at = torch.from_numpy((kept + first[:, None]).astype(np.int64)).to(DEV)
        K, V = [], []
        for l in range(case["layers"]):
            k, v = _kv(case, seed, l)
            K.append(k[at])
            V.append(v[at])
        return {"kept": kept, "mass": np.take_along_axis(m, kept.astype(np.int64), 1), "K": torch.stack(K),
                "V": torch.stack(V)}
    K, V = _kv(case, seed, 0)
    q = _q(case, seed)
    kv, group, hd = case["kv"], case["group"], case["hd"]
    o = torch.empty(q.shape, dtype=torch.float64, device=DEV)
    mass = torch.zeros((len(seqs), max(lens)), dtype=torch.float64, device=DEV)
    r0 = k0 = 0
    for i, (total, rows) in enumerate(seqs):
        index = torch.arange(total, device=DEV)
        for h in range(kv * group):
            kh = K[k0:k0 + total, h // group].double()
            vh = V[k0:k0 + total, h // group].double()
            for a in range(0, rows, 512):  # rows of a prompt, some at a time
                b = min(rows, a + 512)
                z = q[r0 + a:r0 + b, h].double() @ kh.t().contiguous() / hd ** 0.5
                age = (total - rows + torch.arange(a, b, device=DEV))[:, None] - index[None, :]
                hidden = age < 0
                if case["window"]:
                    hidden |= (age >= case["window"]) & (index[None, :] >= case["sinks"])
                w = torch.softmax(z.masked_fill(hidden, -math.inf), dim=1)
                o[r0 + a:r0 + b, h] = w @ vh
                mass[i, :total] += w.sum(dim=0)
        r0 += rows
        k0 += total
    return {"o": o, "mass": mass} if case["mass"] else {"o": o}
