"""The 4-bit cache on the device: what slots hold, attention over it against float64
over the values that it stands for, and the rows of a QKV projection into either
cache."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import mx4_case as mx  # noqa: E402
from cache_case import BLOCK, Cache, bf16, check  # noqa: E402
from mx4_case import Cache4, check_rows, turned  # noqa: E402

pytestmark = pytest.mark.gpu

SPANS = [(0, 0), (1, 0), (1, 5), (16, 4), (17, 16), (40, 33), (256, 4), (1000, 100)]


@pytest.mark.parametrize("kv,hd", [(1, 64), (3, 64), (1, 128), (8, 128)])
def test_slots_hold_what_was_written(kv, hd):
    print(f"[gpu] kv4 slots kv={kv} hd={hd}", flush=True)
    c = Cache4(kv, 2, hd, [1, 16, 17, 200, 45], layers=2, seed=kv + hd, scale=3.0)
    for l in range(2):
        for s in range(5):
            k, v = c.read(l, s)
            np.testing.assert_array_equal(k, c.K[l][s])
            np.testing.assert_array_equal(v, c.V[l][s])
    # a token written again changes no other, nor a slot outside the pool anything
    before = [c.read(1, s) for s in range(5)]
    slots = np.array([c.slots(3, 200)[77], -1, c.n_blocks * 16, c.slots(4, 45)[44]], np.int32)
    k, v = bf16(c.rng.standard_normal((4, kv, hd))), bf16(c.rng.standard_normal((4, kv, hd)))
    sd, kd, vd = torch.from_numpy(slots).cuda(), k.cuda(), v.cuda()
    c.eng.kv4_write(1, sd.data_ptr(), 4, kd.data_ptr(), vd.data_ptr(), c.sp)
    for (s, at), i in (((3, 77), 0), ((4, 44), 3)):
        before[s][0][at], before[s][1][at] = mx.values(k.float().numpy()[i]), mx.values(v.float().numpy()[i])
    for s in range(5):
        for a, b in zip(c.read(1, s), before[s]):
            np.testing.assert_array_equal(a, b)
        np.testing.assert_array_equal(c.read(0, s)[0], c.K[0][s])
    c.close()


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_a_token_that_is_not_finite(bad):
    """Its block of 32 dims reads as NaN; only rows that see it are not finite."""
    for hd in (64, 128):
        c = Cache4(2, 4, hd, [60, 90], seed=3)
        for x in (c.K, c.V):
            x[0][0][30, 1, 5] = bad
            x[0][1][10, 0, hd - 1] = bad
        for s in range(2):
            c.write(0, s)
            k, v = c.read(0, s)
            np.testing.assert_array_equal(k, c.K[0][s])
            np.testing.assert_array_equal(v, c.V[0][s])
        assert np.isnan(c.K[0][0][30, 1, :32]).all() and not np.isnan(c.K[0][0][30, 0]).any()
        c.batch([0, 1], [40, 1])
        c.attend(window=20)
        o = c.out().reshape(41, 2, 4, hd)
        # row i of sequence 0 is at index 20 + i and sees 1 + i .. 20 + i
        sees = np.array([1 + i <= 30 <= 20 + i for i in range(40)])
        assert np.isnan(o[:40][sees][:, 1]).all() and np.isfinite(o[:40][~sees]).all() and np.isfinite(o[:40, 0]).all()
        assert np.isfinite(o[40]).all()
        c.close()


@pytest.mark.parametrize("kv,group,hd", [(1, 1, 64), (2, 16, 64), (4, 3, 128), (8, 4, 128), (3, 7, 128), (1, 16, 128)])
@pytest.mark.parametrize("window,sinks", SPANS)
def test_single_tokens(kv, group, hd, window, sinks):
    print(f"[gpu] kv4 decode kv={kv} group={group} hd={hd} window={window} sinks={sinks}", flush=True)
    c = Cache4(kv, group, hd, [1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 129, 300, 777], seed=kv * 100 + group)
    c.batch(range(13), [1] * 13)
    c.attend(window=window, sinks=sinks)
    check(c, window, sinks)
    c.close()


@pytest.mark.parametrize("bps", [0, 8, 16, 512])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 4), (1500, 130)])
def test_single_tokens_split_and_joined(bps, window, sinks):
    print(f"[gpu] kv4 splits bps={bps} window={window} sinks={sinks}", flush=True)
    c = Cache4(2, 4, 128, [2000, 5, 1023, 1537, 4099], seed=3)
    c.eng.set_tuning(0, bps)
    c.batch(range(5), [1] * 5)
    for _ in range(2):
        c.o.fill_(-7.0)
        c.attend(window=window, sinks=sinks)
        check(c, window, sinks)
    c.close()


@pytest.mark.parametrize("kv,group,hd", [(1, 1, 64), (2, 16, 64), (2, 3, 128), (4, 4, 128), (1, 7, 128)])
@pytest.mark.parametrize("window,sinks", SPANS)
def test_prompt_rows(kv, group, hd, window, sinks):
    print(f"[gpu] kv4 prompt kv={kv} group={group} hd={hd} window={window} sinks={sinks}", flush=True)
    c = Cache4(kv, group, hd, [2, 16, 37, 130, 411, 290], seed=kv * 10 + group)
    c.batch(range(6), [2, 16, 37, 33, 200, 1])
    c.attend(window=window, sinks=sinks)
    check_rows(c, window, sinks)
    c.close()


def test_prompt_rows_of_many_work_items():
    """More work items than compute units (four waves each), and one a row."""
    c = Cache4(4, 4, 64, [300, 513, 700, 90] * 5, seed=11)
    c.batch(range(20), [300, 200, 333, 1] * 5)
    for window, sinks in [(0, 0), (100, 7)]:
        c.attend(window=window, sinks=sinks)
        check_rows(c, window, sinks)
    c.close()
    c = Cache4(2, 4, 128, [70, 300], seed=5)
    c.eng.set_tuning(6, 0)
    c.batch([0, 1], [70, 3])
    for window, sinks in [(0, 0), (20, 3)]:
        c.attend(window=window, sinks=sinks)
        check_rows(c, window, sinks)
    c.close()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("e", [-126, -90, -40, -25, -24, -23, 10, 11, 12, 30, 100])
def test_values_of_any_exponent(hd, e):
    """Values of 2^e and near it, in every block, in some, and beside ordinary ones."""
    print(f"[gpu] kv4 exponents hd={hd} e={e}", flush=True)
    c = Cache4(2, 4, hd, [37, 130, 400], seed=hd + e + 200)
    v = c.V[0]
    v[0] = v[0] * 2.0 ** e
    v[1][:, 1] = v[1][:, 1] * 2.0 ** e
    v[1][20:90:7, 0, :32] = 0
    v[2][64:170] = v[2][64:170] * 2.0 ** e
    for s in range(3):
        v[s] = bf16(v[s]).float().numpy()  # (the smallest bf16 has no bits to spare)
        c.write(0, s)
    for q_lens in ([37, 130, 400], [20, 33, 300], [1, 1, 1]):
        for window, sinks in [(0, 0), (12, 0), (100, 3)]:
            c.batch(range(3), q_lens)
            c.attend(window=window, sinks=sinks)
            check_rows(c, window, sinks)
    c.close()


def test_many_small_weights_keep_their_sum():
    """One key of a score 14 to 19 above all others, of 16,000: they weigh 2^-20 to 2^-27
    each, which a plain fp16 would round to one side or lose."""
    c = Cache4(1, 1, 128, [16000], seed=2)
    c.K[0][0][:] = 0
    c.K[0][0][4000, 0, 0] = 4.0
    c.V[0][0] = np.abs(c.V[0][0])
    c.V[0][0][4000] = 0
    c.write(0, 0)
    c.batch([0], [64])
    c.q[:] = 0
    # scores are divided by sqrt(128)
    c.q[:, 0, 0] = torch.linspace(14, 19, 64).to(c.q.dtype) * 128 ** 0.5 / 4
    c.qd.copy_(c.q)
    c.attend()
    check_rows(c)
    c.close()


def test_long_cache():
    for hd in (64, 128):
        c = Cache4(1, 2, hd, [16384, 16383], seed=6)
        for q_lens in ([1, 1], [3, 40]):
            c.batch([0, 1], q_lens)
            for window, sinks in [(0, 0), (9000, 70)]:
                c.attend(window=window, sinks=sinks)
                check_rows(c, window, sinks)
        c.close()


def test_blocks_behind_four_gigabytes():
    lens, spare = [100, 40, 700], 260000
    need = [-(-n // BLOCK) for n in lens]
    last = sum(need) + spare
    tables, at = [], last
    for n in need:
        tables.append(np.arange(at - n, at)[::-1])
        at -= n
    c = Cache4(8, 2, 128, lens, seed=13, spare=spare, tables=tables)
    assert c._pool4.numel() > 2 ** 32
    for s in range(3):
        K, V = c.read(0, s)
        np.testing.assert_array_equal(K, c.K[0][s])
        np.testing.assert_array_equal(V, c.V[0][s])
    for q_lens in ([1, 1, 1], [60, 1, 37]):
        c.batch([0, 1, 2], q_lens)
        for window, sinks in [(0, 0), (64, 4)]:
            c.attend(window=window, sinks=sinks)
            check_rows(c, window, sinks)
    c.close()


def test_a_shared_prefix_is_the_same_attention():
    c = Cache4(2, 4, 128, [200, 150, 170], seed=7)
    free = [b for b in range(c.n_blocks) if all(b not in t for t in c.blocks)]
    for i, n in ((3, 160), (4, 149)):
        own = -(-(n - 144) // BLOCK)
        c.eng.seq_create(i)
        c.eng.seq_set_blocks(i, np.concatenate([c.blocks[0][:9], free[:own]]).astype(np.int32), n)
        free = free[own:]
        for x in (c.K, c.V):
            x[0].append(np.concatenate([x[0][0][:144], x[0][1][:n - 144]]))
        c.write(0, i, 144)
    c.batch([0, 1, 3, 2, 4], [1] * 5)
    for window, sinks in [(0, 0), (30, 5)]:
        c.attend(window=window, sinks=sinks)
        check(c, window, sinks)
    c.close()


def test_slots_behind_a_sequence_do_not_matter():
    """Codes and exponents of no token: the pool starts as exponents that say NaN."""
    for hd in (64, 128):
        c = Cache4(2, 4, hd, [5, 33, 100], seed=12)
        for ql in ([1, 1, 1], [5, 20, 99]):
            c.batch([0, 1, 2], ql)
            c.attend()
            check_rows(c)
        c.close()


def test_large_scores():
    c = Cache4(2, 4, 128, [300, 90], seed=8, scale=2.0 ** 20)
    for ql in ([1, 1], [100, 90]):
        c.batch([0, 1], ql)
        c.attend()
        assert np.isfinite(c.out()).all()
    c.close()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_a_query_that_is_not_finite(hd, bad):
    """Only its own row and head are not finite."""
    c = Cache4(2, 4, hd, [90, 300, 1500], seed=31)
    for q_lens in ([60, 33, 1], [1, 1, 1]):
        c.batch([0, 1, 2], q_lens)
        c.attend(window=200, sinks=4)
        finite = c.out()
        rows = [0, sum(q_lens) - 1, sum(q_lens) // 2]
        for r in rows:
            c.qd[r, 5, 40] = bad
        c.attend(window=200, sinks=4)
        got = c.out()
        for r in rows:
            assert not np.isfinite(got[r, 5]).any()
            got[r, 5] = finite[r, 5]
        c.out = lambda: got
        check_rows(c, 200, 4)
        del c.out
    c.close()


def test_replayed_beside_eager_calls():
    c = Cache4(2, 4, 128, [300, 97, 1500], seed=9)
    c.batch([0, 1, 2], [60, 1, 1])
    c.attend()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        c.attend(window=200, sinks=4, stream=torch.cuda.current_stream().cuda_stream)
    for i in range(3):
        c.q = bf16(c.rng.standard_normal(tuple(c.q.shape)))
        c.qd.copy_(c.q)
        c.o[:-1].fill_(0)
        g.replay()
        check_rows(c, 200, 4)
        c.attend()
        check_rows(c)
    c.close()


# ------------------------------------------------------------------ rows of a QKV projection
def _rows(cls, kv, group, hd, lens, q_lens, seed, pad=0, max_pos=16384):
    c = cls(kv, group, hd, lens, layers=2, seed=seed, max_pos=max_pos)
    c.batch(range(len(lens)), q_lens)
    rows, width = sum(q_lens), kv * (group + 2) * hd
    x = bf16(c.rng.standard_normal((rows, width + pad)) * 2.0)
    gains = bf16(1 + 0.3 * c.rng.standard_normal((2, hd)))
    nb = c.eng.rope_bytes()
    c._rope, at = c.buf(nb, "cuda")
    c.eng.rope_bind(at, nb, c.sp)
    return c, x, gains


def _check_rows(c, x, gains, bits, norm, layer=1):
    kv, heads, hd = c.kv, c.kv * c.group, c.hd
    rows = x.shape[0]
    xd, gd = x.cuda(), gains.cuda()
    q = torch.full((rows + 1, heads, hd), -7.0, dtype=torch.bfloat16, device="cuda")
    c.eng.qkv_norm_rope(layer, xd.data_ptr(), x.shape[1], gd[0].data_ptr() if norm[0] else None,
                        gd[1].data_ptr() if norm[1] else None, q.data_ptr(), bits, c.sp)
    h = c.eng.batch_host()
    slots = torch.from_numpy(h["slot"]).cuda()
    K = torch.zeros((rows, kv, hd), dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    (c.eng.kv4_read if bits == 4 else c.eng.kv_read)(layer, slots.data_ptr(), rows, K.data_ptr(), V.data_ptr(), c.sp)
    torch.cuda.synchronize()
    assert (q[-1] == -7).all()
    q, K, V = (t.float().cpu().numpy().astype(np.float64) for t in (q[:-1], K, V))
    xs = x[:, :kv * (c.group + 2) * hd].float().numpy().astype(np.float64).reshape(rows, -1, hd)
    pos = h["pos"].astype(np.float64)
    g = gains.float().numpy().astype(np.float64)
    eps, theta = float(np.float32(1e-5)), 500000.0
    wq, mq = turned(xs[:, :heads], pos, g[0] if norm[0] else None, theta, eps)
    wk, mk = turned(xs[:, heads:heads + kv], pos, g[1] if norm[1] else None, theta, eps)
    # float32: a sum of squares (hd / 8 + 6 roundings), a root, a quotient, two products,
    # cos and sin (one each) and the turn (two): at most 40 half steps; half a step of bf16
    near = lambda got, want, mag: (np.abs(got - want) <= 40 * 2.0 ** -24 * mag + 2.0 ** -8 * np.abs(want) + 1e-38).all()
    assert near(q, wq, mq)
    wv = xs[:, heads + kv:]
    if bits == 16:
        assert near(K, wk, mk)
        np.testing.assert_array_equal(V, wv)
    else:
        # (keys are taken in 64 bits: their codes are the exact values')
        np.testing.assert_array_equal(K, mx.values(wk))
        np.testing.assert_array_equal(V, mx.values(wv))
    return h["slot"]


@pytest.mark.parametrize("kv,group,hd", [(1, 1, 64), (3, 2, 64), (2, 16, 64), (8, 4, 128), (1, 3, 128), (5, 7, 128)])
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("norm", [(True, True), (False, False), (False, True), (True, False)])
def test_qkv_rows(kv, group, hd, bits, norm):
    print(f"[gpu] qkv rows kv={kv} group={group} hd={hd} bits={bits} norm={norm}", flush=True)
    c, x, gains = _rows(Cache4 if bits == 4 else Cache, kv, group, hd, [1, 40, 333, 2000], [1, 1, 47, 130], kv * 7 + hd, pad=24)
    written = set(_check_rows(c, x, gains, bits, norm).tolist())
    # nothing else of the cache has changed, in this layer or the other
    for layer in range(2):
        for s, n in enumerate(c.lens):
            k, v = c.read(layer, s)
            keep = np.array([layer == 0 or int(t) not in written for t in c.slots(s, n)])
            np.testing.assert_array_equal(k[keep], c.K[layer][s][keep])
            np.testing.assert_array_equal(v[keep], c.V[layer][s][keep])
    c.close()


@pytest.mark.parametrize("bits", [16, 4])
def test_qkv_rows_last_positions_and_evicted_ones(bits):
    c, x, gains = _rows(Cache4 if bits == 4 else Cache, 2, 2, 128, [16384, 16383], [70, 1], 5)
    _check_rows(c, x, gains, bits, (True, True))
    c.close()
    if bits == 16:  # a shorter cache whose positions go on
        c, _, gains = _rows(Cache, 2, 2, 64, [300], [1], 6)
        mass = torch.rand((1, 300), device="cuda")
        c.eng.seq_create(9)
        nb = c.eng.kv_evict_bytes([0], [100])
        meta, at = c.buf(nb, "cuda")
        kept = torch.empty((1, 100), dtype=torch.int32, device="cuda")
        c.eng.kv_evict([9], [0], [100], 4, 20, mass.data_ptr(), 300, at, nb, kept_ptr=kept.data_ptr(), out_stride=100, stream=c.sp)
        c.eng.reserve(9, 3)
        c.batch([9], [3])
        assert c.eng.batch_host()["pos"].tolist() == [300, 301, 302]
        _check_rows(c, bf16(c.rng.standard_normal((3, 2 * 4 * 64))), gains, 16, (True, True))
        c.close()


def test_qkv_rows_refusals():
    c, x, gains = _rows(Cache4, 2, 2, 64, [40, 30], [3, 1], 4, max_pos=64)
    from paper_2609_37062_amd import vsk
    xd = x.cuda()
    q = torch.zeros((4, 4, 64), dtype=torch.bfloat16, device="cuda")
    ok = dict(layer=0, qkv=xd.data_ptr(), stride=x.shape[1], q=q.data_ptr(), bits=4, gq=None)
    for bad, code in ((dict(layer=2), "RANGE"), (dict(layer=-1), "RANGE"), (dict(qkv=None), "ARG"), (dict(q=None), "ARG"),
                      (dict(stride=x.shape[1] - 8), "ARG"), (dict(stride=x.shape[1] + 4), "ARG"), (dict(stride=1 << 62), "ARG"),
                      (dict(qkv=xd.data_ptr() + 8), "ARG"), (dict(q=q.data_ptr() + 8), "ARG"), (dict(bits=8), "ARG"),
                      (dict(gq=gains.data_ptr() | 1), "ARG"), (dict(q=xd.data_ptr() + 64), "ARG")):
        a = {**ok, **bad}
        with pytest.raises(vsk.VskError) as e:
            c.eng.qkv_norm_rope(a["layer"], a["qkv"], a["stride"], a["gq"], None, a["q"], a["bits"], c.sp)
        assert e.value.code == code, bad
    for bad, code in ((dict(q=c.qd.data_ptr() + 8), "ARG"), (dict(o=c.qd.data_ptr()), "ARG"), (dict(layer=2), "RANGE"),
                      (dict(window=-1), "ARG"), (dict(sinks=-1), "ARG"), (dict(ws=c.ws + 256), "STATE"), (dict(q=None), "ARG")):
        a = {**dict(layer=0, q=c.qd.data_ptr(), o=c.o.data_ptr(), window=0, sinks=0, ws=c.ws), **bad}
        with pytest.raises(vsk.VskError) as e:
            c.eng.kv4_attend(a["layer"], a["q"], a["o"], a["ws"], c.ws_bytes, a["window"], a["sinks"], c.sp)
        assert e.value.code == code, bad
    c.close()


@pytest.mark.parametrize("cls", [Cache, Cache4])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,q_len", [(700, 5), (700, 1), (16000, 3), (16000, 1), (16000, 200)])
def test_equal_scores_weigh_the_same_at_any_size(cls, hd, n, q_len):
    """Scores of 2^12 to 2^29.  Two keys A and B have the same one, some units in its last
    place above a third's, L, and every other key's is zero (no weight at all).  What L
    weighs is the arithmetic's; A and B weigh the same, and V is 2 at L, 3 at A, 1 at B
    (all exact in 4 bits): 2 throughout, wherever the three stand and whichever is the
    first to set a walk's maximum."""
    print(f"[gpu] equal scores {cls.__name__} hd={hd} n={n} q_len={q_len}", flush=True)
    kv, group = 4, 4
    c = cls(kv, group, hd, [n], seed=17)
    K, V = c.K[0][0], c.V[0][0]
    K[:] = 0
    far = n // 700
    # (L and one of A and B in the same steps' part of a prompt row's walk, or in none)
    for h, (l, a, b) in enumerate(((3, 197, 360 * far), (40, 70 * far, 104), (2, 600 * far, 600 * far + 1), (97 * far, 10, 97 * far + 64))):
        K[[l, a, b], h, 0] = 2.0 ** 14
        K[[a, b], h, 32] = 1.0
        V[[l, a, b], h] = np.array([2.0, 3.0, 1.0])[:, None]
    c.write(0, 0)
    np.testing.assert_array_equal(c.read(0, 0)[0], K)
    c.batch([0], [q_len])
    c.q[:] = 0
    for e in range(-2, 16):
        for units in (1, 2, 3, 4, 6):
            # a score of 2^(14 + e), whose last place is 2^(e - 9)
            c.q[:, :, 0] = 2.0 ** e
            c.q[:, :, 32] = units * 2.0 ** (e - 9)
            c.qd.copy_(c.q)
            c.attend()
            # a weight is off by at most 2^-11 of itself (half a step of fp16) and some
            # steps of float32, of values up to 3; half a step of bf16 of 2
            err = np.abs(c.out() - 2.0)
            assert (err <= 2.0 ** -7 + 3 * 2.0 ** -11 + 3 * 2.0 ** -16).all(), (e, units, float(err.max()), np.argwhere(~(err <= 2.0 ** -6))[:4].tolist())
    c.close()


@pytest.mark.parametrize("cls", [Cache, Cache4])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("q_len", [1, 3, 70])
def test_keys_that_are_not_finite_fill_a_split(cls, hd, q_len):
    """3,840 keys in a row that are NaN: whole splits of one (of 256, 320, 384, 640 or 768
    keys).  Every row sees them, so every output of their head is NaN, and no other."""
    print(f"[gpu] a split of NaN {cls.__name__} hd={hd} q_len={q_len}", flush=True)
    c = cls(2, 4, hd, [16000], seed=23)
    c.K[0][0][:3840, 1] = np.nan
    c.write(0, 0)
    c.batch([0], [q_len])
    c.attend()
    o = c.out().reshape(q_len, 2, 4, hd)
    assert np.isnan(o[:, 1]).all()
    assert np.isfinite(o[:, 0]).all()
    c.attend(window=9000)  # (none of them is seen)
    assert np.isfinite(c.out()).all()
    c.close()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("q_lens", [[1, 1, 1], [5, 20, 99], [2, 33, 40]])
def test_slots_of_no_token_leave_no_bit(hd, q_lens):
    """The same tokens in a pool that held other things before: the same bits."""
    print(f"[gpu] unused slots hd={hd} q_lens={q_lens}", flush=True)
    c = Cache4(2, 4, hd, [5, 33, 100], seed=12)
    c.batch([0, 1, 2], q_lens)
    outs = []
    for fill in (0x7f, 0xff, 0x00, 0x97, None):  # exponents 0, NaN, -127, 24, drawn ones
        if fill is None:
            c._pool4.view(torch.uint8).copy_(torch.from_numpy(np.random.default_rng(5).integers(0, 256, c._pool4.view(torch.uint8).numel(), np.uint8)))
        else:
            c._pool4.view(torch.uint8).fill_(fill)
        for s in range(3):
            c.write(0, s)
        for window, sinks in [(0, 0), (12, 3)]:
            c.o[:-1].fill_(0)
            c.attend(window=window, sinks=sinks)
            check_rows(c, window, sinks)
            outs.append(c.out())
    for i in range(2, len(outs)):
        np.testing.assert_array_equal(outs[i], outs[i % 2])
    c.close()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("norm", [(True, True), (False, False)])
def test_qkv_rows_of_any_magnitude(hd, bits, norm):
    """Heads whose squares a float32 does not hold, and tiny ones."""
    print(f"[gpu] qkv rows of any magnitude hd={hd} bits={bits} norm={norm}", flush=True)
    c, x, gains = _rows(Cache4 if bits == 4 else Cache, 2, 3, hd, [40, 333], [33, 20], 77)
    e = torch.from_numpy(c.rng.choice([-126, -80, -64, 0, 50, 62, 64, 66, 90, 120, 124], (53, 10)))
    # (heads of mixed size too: half of the dims 2^-30 of the others)
    f = torch.ones(hd, dtype=torch.float64)
    f[::2] = 2.0 ** -30
    v = x.reshape(53, 10, hd).double() * 2.0 ** e.double()[:, :, None]
    v[::3] *= f
    x = v.to(torch.bfloat16).reshape(53, -1)
    assert torch.isfinite(x).all()
    _check_rows(c, x, gains, bits, norm)
    c.close()


@pytest.mark.parametrize("bits", [16, 4])
def test_qkv_rows_without_an_epsilon(bits, monkeypatch):
    """Tiny heads are normed as they are where nothing is added to their squares."""
    import cache_case
    model = cache_case.model

    def no_eps(*a, **k):
        m = model(*a, **k)
        m.rms_eps = 0.0
        return m

    monkeypatch.setattr(cache_case, "model", no_eps)
    c, x, gains = _rows(Cache4 if bits == 4 else Cache, 2, 3, 128, [40], [40], 78)
    e = torch.from_numpy(c.rng.choice([-100, -75, -60, -44, 0, 70], (40, 10)))
    x = (x.reshape(40, 10, 128).double() * 2.0 ** e.double()[:, :, None]).to(torch.bfloat16).reshape(40, -1)
    xd, gd = x.cuda(), gains.cuda()
    q = torch.zeros((40, 6, 128), dtype=torch.bfloat16, device="cuda")
    c.eng.qkv_norm_rope(1, xd.data_ptr(), x.shape[1], gd[0].data_ptr(), gd[1].data_ptr(), q.data_ptr(), bits, c.sp)
    K, _ = c.read(1, 0)
    xs, g = x.double().numpy().reshape(40, -1, 128), gains.double().numpy()
    pos = c.eng.batch_host()["pos"].astype(np.float64)
    wq, mq = turned(xs[:, :6], pos, g[0], 500000.0, 0.0)
    wk, mk = turned(xs[:, 6:8], pos, g[1], 500000.0, 0.0)
    # (as in _check_rows)
    near = lambda got, want, mag: (np.abs(got - want) <= 40 * 2.0 ** -24 * mag + 2.0 ** -8 * np.abs(want)).all()
    assert near(q.double().cpu().numpy(), wq, mq)
    if bits == 16:
        assert near(K.astype(np.float64), wk, mk)
    else:
        np.testing.assert_array_equal(K, mx.values(wk))
    c.close()
