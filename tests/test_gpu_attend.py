"""vsk_attend on the device against float64: single tokens and prompt rows, full
and windowed, one split and several, every head layout, values that are not
finite where a row does not see them, and the weight per cached token."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from cache_case import BLOCK, Cache, attend_ref, check, visible  # noqa: E402

pytestmark = pytest.mark.gpu

SPANS = [(0, 0), (1, 0), (1, 5), (16, 4), (17, 16), (40, 33), (256, 4), (1000, 100)]


@pytest.mark.parametrize("kv,group,hd", [(1, 1, 64), (2, 16, 64), (4, 3, 128), (8, 4, 128), (3, 7, 128), (1, 16, 128)])
@pytest.mark.parametrize("window,sinks", SPANS)
def test_single_tokens(kv, group, hd, window, sinks):
    print(f"[gpu] attend decode kv={kv} group={group} hd={hd} window={window} sinks={sinks}", flush=True)
    c = Cache(kv, group, hd, [1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 129, 300, 777], seed=kv * 100 + group)
    c.batch(range(13), [1] * 13)
    c.attend(window=window, sinks=sinks)
    check(c, window, sinks)
    c.close()


@pytest.mark.parametrize("bps", [0, 8, 16, 512])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 4), (1500, 130)])
def test_single_tokens_split_and_joined(bps, window, sinks):
    print(f"[gpu] attend splits bps={bps} window={window} sinks={sinks}", flush=True)
    c = Cache(2, 4, 128, [2000, 5, 1023, 1537, 4099], seed=3)
    c.eng.set_tuning(0, bps)
    c.batch(range(5), [1] * 5)
    for _ in range(2):  # the second call finds the arrival counters at zero again
        c.o.fill_(-7.0)
        c.attend(window=window, sinks=sinks)
        check(c, window, sinks)
    c.close()


@pytest.mark.parametrize("kv,group,hd", [(1, 1, 64), (2, 16, 64), (2, 3, 128), (4, 4, 128), (1, 7, 128)])
@pytest.mark.parametrize("window,sinks", SPANS)
def test_prompt_rows(kv, group, hd, window, sinks):
    print(f"[gpu] attend prompt kv={kv} group={group} hd={hd} window={window} sinks={sinks}", flush=True)
    c = Cache(kv, group, hd, [2, 16, 37, 130, 411, 290], seed=kv * 10 + group)
    c.batch(range(6), [2, 16, 37, 33, 200, 1])  # fresh, later chunks, and one decode row
    c.attend(window=window, sinks=sinks)
    check(c, window, sinks)
    c.close()


def test_prompt_rows_one_work_item_a_row():
    c = Cache(2, 4, 128, [70, 300], seed=5)
    c.eng.set_tuning(6, 0)
    c.batch([0, 1], [70, 3])
    for window, sinks in [(0, 0), (20, 3)]:
        c.attend(window=window, sinks=sinks)
        check(c, window, sinks)
    c.close()


def test_long_cache():
    """16384 cached tokens: 1024 blocks, single tokens and a prompt's last rows."""
    c = Cache(1, 2, 64, [16384, 16383], seed=6)
    for q_lens in ([1, 1], [3, 40]):
        c.batch([0, 1], q_lens)
        for window, sinks in [(0, 0), (9000, 70)]:
            c.attend(window=window, sinks=sinks)
            check(c, window, sinks)
    c.close()


def test_a_shared_prefix_is_the_same_attention():
    """Sequences whose tables start with the same blocks, decoding."""
    c = Cache(2, 4, 128, [200, 150, 170], seed=7, tables=None, spare=64)
    # sequences 3, 4 hold sequence 0's first 9 blocks and own blocks behind them
    free = [b for b in range(c.n_blocks) if all(b not in t for t in c.blocks)]
    for i, n in ((3, 160), (4, 149)):
        own = -(-(n - 144) // BLOCK)
        c.eng.seq_create(i)
        c.eng.seq_set_blocks(i, np.concatenate([c.blocks[0][:9], free[:own]]).astype(np.int32), n)
        free = free[own:]
        k = np.concatenate([c.K[0][0][:144], c.K[0][1][:n - 144]])
        v = np.concatenate([c.V[0][0][:144], c.V[0][1][:n - 144]])
        c.K[0].append(k)
        c.V[0].append(v)
        c.write(0, i, 144)
    c.batch([0, 1, 3, 2, 4], [1] * 5)
    assert c.eng.batch_prefix_info()[1] == 1
    mass = torch.zeros((5, 256), device="cuda")
    for window, sinks in [(0, 0), (30, 5)]:
        c.attend(window=window, sinks=sinks, mass=mass)
        check(c, window, sinks, mass=mass)
    c.close()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("prompt", [False, True])
def test_what_a_row_does_not_see_does_not_matter(bad, prompt):
    """K and V that are not finite: hidden by the window, or only visible to
    later rows, whose outputs are then not finite."""
    print(f"[gpu] attend bad={bad} prompt={prompt}", flush=True)
    window, sinks = 40, 5
    c = Cache(2, 4, 128, [300, 97], seed=8)
    ql = [60, 50] if prompt else [1, 1]
    c.batch([0, 1], ql)
    c.attend(window=window, sinks=sinks)
    good = c.out()
    mass = torch.zeros((2, 300), device="cuda")
    # hidden from every row: behind the sinks, before the first row's window
    for s in (0, 1):
        n = len(c.K[0][s])
        lo = n - ql[s] - window
        if lo > 8:
            c.K[0][s][5:lo] = bad
            c.V[0][s][5:lo] = bad
            c.write(0, s)
    c.attend(window=window, sinks=sinks, mass=mass)
    np.testing.assert_array_equal(c.out(), good)
    m = mass.cpu().numpy()
    assert np.isfinite(m).all() and (m[0, 5:300 - ql[0] - window] == 0).all()
    if prompt:
        # one key of the chunk itself: rows before it, and rows whose window has
        # left it behind, do not see it
        key = 300 - 60 + 7
        for which in (c.V, c.K):
            keep = which[0][0][key].copy()
            which[0][0][key] = bad
            c.write(0, 0)
            c.attend(window=window, sinks=sinks)
            o = c.out()
            for r in range(60):
                p = 240 + r
                if not visible(p, 300, window, sinks)[key]:
                    np.testing.assert_array_equal(o[r], good[r], err_msg=str(r))
                elif which is c.V:
                    assert not np.isfinite(o[r]).any(), r
            which[0][0][key] = keep
            c.write(0, 0)
    c.close()


@pytest.mark.parametrize("q_lens", [[1, 1, 1, 1], [1, 40, 17, 2], [300, 33, 200, 1]])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (20, 3), (100, 40)])
def test_weights_per_token(q_lens, window, sinks):
    print(f"[gpu] attend mass q_lens={q_lens} window={window} sinks={sinks}", flush=True)
    c = Cache(4, 3, 64, [300, 40, 217, 33], seed=9)
    c.batch(range(4), q_lens)
    mass = torch.full((4, 333), 0.5, device="cuda")
    c.attend(window=window, sinks=sinks, mass=mass)
    ref = check(c, window, sinks, mass=mass)
    m = mass.cpu().numpy()
    for i, n in enumerate(c.lens):
        assert (m[i, n:] == 0.5).all(), "entries behind the sequence"
        assert abs(m[i, :n].sum() - q_lens[i] * 12) < 1e-3 * q_lens[i] * 12  # every row and head gives 1
        assert ref[i][1].shape == (n,)
    base = mass.cpu().numpy().astype(np.float64)
    c.attend(window=window, sinks=sinks, mass=mass, add=True)
    check(c, window, sinks, mass=mass, base=base)
    again = torch.zeros_like(mass)
    c.attend(window=window, sinks=sinks, mass=again)
    third = torch.zeros_like(mass)
    c.attend(window=window, sinks=sinks, mass=third)
    assert torch.equal(again, third), "the same sums on every call"
    c.close()


def test_weights_without_room_for_scores_or_parts():
    """So long and so few rows that the workspace holds neither the scores nor
    the parts of the weights: they are taken as 32 keys a workgroup."""
    c = Cache(1, 1, 64, [16001, 15000, 16384, 16383], seed=13)
    c.batch(range(4), [2, 1, 1, 1])
    mass = torch.zeros((4, 16384), device="cuda")
    for window, sinks in [(0, 0), (5000, 33)]:
        c.attend(window=window, sinks=sinks, mass=mass)
        check(c, window, sinks, mass=mass)
    c.close()


def test_large_scores_stay_finite():
    """Scores of 2^26: one key takes all the weight."""
    c = Cache(2, 4, 128, [200, 90], seed=10, scale=2.0 ** 24)
    c.batch([0, 1], [40, 1])
    mass = torch.zeros((2, 200), device="cuda")
    for window, sinks in [(0, 0), (30, 2)]:
        c.attend(window=window, sinks=sinks, mass=mass)
        o = c.out()
        assert np.isfinite(o).all()
        r0 = 0
        for i, ql in enumerate(c.q_lens):
            n = c.lens[i]
            q = c.q[r0:r0 + ql].double().numpy()
            for r in range(ql):
                see = np.flatnonzero(visible(n - ql + r, n, window, sinks))
                for h in range(8):
                    s = c.K[0][i][see, h // 4].astype(np.float64) @ q[r, h]
                    top = np.sort(s)[-2:] if len(see) > 1 else np.array([-np.inf, s[0]])
                    if top[1] - top[0] < 2.0 ** 14:  # (float32 sums tell these apart)
                        continue
                    np.testing.assert_array_equal(o[r0 + r, h], c.V[0][i][see[s.argmax()], h // 4])
            m = mass[i, :n].cpu().numpy()
            assert np.isfinite(m).all() and abs(m.sum() - ql * 8) < 1e-3 * ql * 8
            r0 += ql
    c.close()


def test_layers_streams_and_replays():
    """Each layer reads its own cache; a call on another stream, and one in a
    captured graph, replayed with eager work between, give the same bits."""
    c = Cache(2, 4, 128, [1500, 700, 90], layers=3, seed=11)
    c.batch(range(3), [1, 30, 1])
    eager = []
    for l in range(3):
        c.attend(layer=l, window=333, sinks=4)
        check(c, 333, 4, layer=l)
        eager.append(c.out())
    side = torch.cuda.Stream()
    mass = torch.zeros((3, 1500), device="cuda")
    with torch.cuda.stream(side):
        c.attend(layer=1, window=333, sinks=4, mass=mass, stream=side.cuda_stream)
    np.testing.assert_array_equal(c.out(), eager[1])
    want = mass.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.attend(layer=1, window=333, sinks=4, mass=mass, stream=torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        c.attend(layer=2, window=333, sinks=4)
        np.testing.assert_array_equal(c.out(), eager[2])
        mass.fill_(9.0)
        g.replay()
        np.testing.assert_array_equal(c.out(), eager[1])
        for i, n in enumerate(c.lens):
            assert torch.equal(mass[i, :n], want[i, :n]) and bool((mass[i, n:] == 9.0).all())
    c.close()


def test_heads_of_one_query_each_and_odd_rows():
    """A single row of a single head against the formula written out."""
    c = Cache(1, 1, 128, [50], seed=12)
    c.batch([0], [1])
    c.attend(window=9, sinks=2)
    o, ob, _, _ = attend_ref(c.q.float().numpy(), c.K[0][0], c.V[0][0], 49, 9, 2)
    assert (np.abs(c.out() - o) <= ob).all()
    see = [0, 1] + list(range(41, 50))
    s = c.K[0][0][see, 0].astype(np.float64) @ c.q[0, 0].double().numpy() / np.sqrt(128)
    w = np.exp(s) / np.exp(s).sum()
    np.testing.assert_allclose(o[0, 0], w @ c.V[0][0][see, 0], rtol=1e-12, atol=1e-12)
    c.close()


@pytest.mark.parametrize("kv,group,hd", [(2, 4, 128), (1, 7, 128), (2, 16, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1000, 200), (70, 33)])
def test_few_prompt_rows_behind_long_caches(kv, group, hd, window, sinks):
    """Walks that are cut into splits and joined, beside short ones and a decode
    row, with their weights; and keys behind the chunk that only some rows see."""
    c = Cache(kv, group, hd, [3000, 1700, 901, 40], seed=14)
    c.batch(range(4), [7, 33, 1, 20])
    mass = torch.zeros((4, 3000), device="cuda")
    c.attend(window=window, sinks=sinks, mass=mass)
    check(c, window, sinks, mass=mass)
    good = c.out()
    if window:
        lo, hi = sinks, 3000 - 7 - window  # no row of the first sequence sees these
        if lo < hi:
            for x in (c.K, c.V):
                x[0][0][lo:hi] = np.nan
            c.write(0, 0)
            c.attend(window=window, sinks=sinks, mass=mass)
            np.testing.assert_array_equal(c.out(), good)
            assert bool(torch.isfinite(mass).all()) and bool((mass[0, lo:hi] == 0).all())
    c.V[0][0][2996] = np.inf  # rows 0..2 do not see it
    c.write(0, 0)
    c.attend(window=window, sinks=sinks)
    o = c.out()
    np.testing.assert_array_equal(o[:3], good[:3])
    np.testing.assert_array_equal(o[7:], good[7:])
    assert not np.isfinite(o[3:7]).any()
    c.close()


@pytest.mark.parametrize("hd", [64, 128])
def test_many_short_prompts(hd):
    """More work items than compute units."""
    lens = [2 + 7 * i % 121 + i for i in range(34)]
    c = Cache(8, 2, hd, lens, seed=15)
    c.batch(range(34), [min(n, 2 + i % 4) for i, n in enumerate(lens)])
    mass = torch.zeros((34, max(lens)), device="cuda")
    for window, sinks in [(0, 0), (18, 3)]:
        c.attend(window=window, sinks=sinks, mass=mass)
        check(c, window, sinks, mass=mass)
    c.close()


def test_two_engines_on_two_streams():
    """Calls of different engines, side by side, are what each is alone."""
    cs = [Cache(2, 4, 128, [900, 333], seed=16), Cache(4, 2, 64, [500, 70, 5], seed=17)]
    for c, ql in zip(cs, ([40, 1], [1, 70, 2])):
        c.batch(range(len(c.lens)), ql)
    masses = [torch.zeros((len(c.lens), 900), device="cuda") for c in cs]
    alone = []
    for c, m in zip(cs, masses):
        c.attend(window=100, sinks=9, mass=m)
        alone.append((c.out(), m.clone()))
        m.zero_()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(8):
        for c, m, s in zip(cs, masses, streams):
            c.attend(window=100, sinks=9, mass=m, stream=s.cuda_stream)
    for c, m, (o, am) in zip(cs, masses, alone):
        np.testing.assert_array_equal(c.out(), o)
        assert torch.equal(m, am)
        c.close()


@pytest.mark.parametrize("kv,hd", [(1, 64), (3, 128)])
def test_reading_slots_of_any_order(kv, hd):
    """kv_read: runs of a block and none, the same slot twice, slots outside the
    pool (their rows stay as they are), outputs 2 bytes off, list lengths around 16."""
    c = Cache(kv, 1, hd, [100, 33], seed=18)
    own = np.concatenate([c.slots(0, 100), c.slots(1, 33)])
    K = np.concatenate(c.K[0])
    V = np.concatenate(c.V[0])
    rng = np.random.default_rng(3)
    for order in (np.arange(133), np.arange(5, 133), rng.permutation(133), rng.integers(0, 133, 200), np.arange(16),
                  np.arange(8, 25), np.array([7])):
        for off in (0, 1):
            n = len(order)
            sl = own[order].astype(np.int32)
            skip = rng.random(n) < 0.1
            sl[skip] = rng.choice([-1, c.n_blocks * BLOCK, 2 ** 31 - 1], skip.sum())
            s = torch.from_numpy(sl).cuda()
            k = torch.full((n * kv * hd + 9,), -3.0, dtype=torch.bfloat16, device="cuda")
            v = torch.full_like(k, -3.0)
            c.eng.kv_read(0, s.data_ptr(), n, k.data_ptr() + 2 * off, v.data_ptr() + 2 * off, c.sp)
            torch.cuda.synchronize()
            for got, src in ((k, K), (v, V)):
                want = np.full(n * kv * hd + 9, -3.0, np.float32)
                x = want[off:off + n * kv * hd].reshape(n, kv, hd)
                x[~skip] = src[order[~skip]]
                np.testing.assert_array_equal(got.float().cpu().numpy(), want)
    c.close()


@pytest.mark.parametrize("hd,group", [(64, 2), (128, 1)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (3000, 40)])
def test_single_tokens_of_uneven_long_caches(hd, group, window, sinks):
    """Rows of which some have one split and some many, all of them in one round."""
    c = Cache(8, group, hd, [8000, 300, 5000, 2500, 1200, 40, 1], seed=19)
    c.batch(range(7), [1] * 7)
    mass = torch.zeros((7, 8000), device="cuda")
    c.attend(window=window, sinks=sinks)
    check(c, window, sinks)
    c.attend(window=window, sinks=sinks, mass=mass)
    check(c, window, sinks, mass=mass)
    c.close()


def test_uneven_caches_behind_a_shared_prefix():
    c = Cache(8, 1, 64, [6000], seed=20, spare=600)
    free = [b for b in range(c.n_blocks) if b not in set(c.blocks[0].tolist())]
    rng = np.random.default_rng(4)
    for i, n in enumerate((4000, 500, 900, 2000), start=1):
        own = -(-(n - 320) // BLOCK)
        c.eng.seq_create(i)
        c.eng.seq_set_blocks(i, np.concatenate([c.blocks[0][:20], free[:own]]).astype(np.int32), n)
        free = free[own:]
        perm = 320 + rng.permutation(6000 - 320)[:n - 320]
        c.K[0].append(np.concatenate([c.K[0][0][:320], c.K[0][0][perm]]))
        c.V[0].append(np.concatenate([c.V[0][0][:320], c.V[0][0][perm]]))
        c.write(0, i, 320)
    c.batch(range(5), [1] * 5)
    assert c.eng.batch_prefix_info()[1] == 1
    mass = torch.zeros((5, 6000), device="cuda")
    for window, sinks in [(0, 0), (2500, 16)]:
        c.attend(window=window, sinks=sinks, mass=mass)
        check(c, window, sinks, mass=mass)
    c.close()


def test_many_single_tokens():
    """More rows than a wave counts, and splits of 128 blocks."""
    lens = [1 + 37 * i % 700 + (2500 if i % 23 == 5 else 0) for i in range(97)]
    c = Cache(4, 1, 64, lens, seed=21)
    c.batch(range(97), [1] * 97)
    mass = torch.zeros((97, max(lens)), device="cuda")
    for window, sinks in [(0, 0), (400, 7)]:
        c.attend(window=window, sinks=sinks, mass=mass)
        check(c, window, sinks, mass=mass)
    c.close()


def test_weights_of_prompt_rows_one_work_item_a_row():
    c = Cache(2, 3, 64, [70, 300, 33], seed=22)
    c.eng.set_tuning(6, 0)
    c.batch([0, 1, 2], [70, 5, 1])
    mass = torch.zeros((3, 300), device="cuda")
    for window, sinks in [(0, 0), (20, 3)]:
        c.attend(window=window, sinks=sinks, mass=mass)
        check(c, window, sinks, mass=mass)
    c.close()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("group", [3, 5, 7, 12])
@pytest.mark.parametrize("scale", [60.0, 2.0 ** 24])
def test_weights_of_large_scores_where_groups_leave_columns_over(group, hd, scale):
    """32 columns hold 10, 6, 4, 2 whole rows of these groups.  A row's own key
    may score far above all that the row before it sees; every weight is finite,
    and a row's weights come to 1 a head."""
    for seed in range(3):
        print(f"[gpu] large scores group={group} hd={hd} scale={scale} seed={seed}", flush=True)
        c = Cache(1, group, hd, [40, 33], seed=100 + seed, scale=scale)
        c.batch([0, 1], [40, 33])
        mass = torch.zeros((2, 40), device="cuda")
        for window, sinks in [(0, 0), (1, 0), (30, 2)]:
            c.attend(window=window, sinks=sinks, mass=mass)
            if scale < 2.0 ** 20:
                check(c, window, sinks, mass=mass)
            assert np.isfinite(c.out()).all()
            for i, n in enumerate(c.lens):
                m = mass[i, :n].cpu().numpy()
                assert np.isfinite(m).all(), (window, np.flatnonzero(~np.isfinite(m)))
                assert abs(m.sum() - n * group) < 1e-3 * n * group
        c.close()


@pytest.mark.parametrize("group", [3, 4, 7, 12])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_a_query_that_is_not_a_number_stays_with_the_keys_it_sees(group, window, sinks):
    c = Cache(1, group, 64, [60], seed=23)
    c.batch([0], [45])
    mass = torch.zeros((1, 60), device="cuda")
    q = c.qd.clone()
    for r in range(45):
        c.qd.copy_(q)
        c.qd[r] = float("nan")
        c.attend(window=window, sinks=sinks, mass=mass)
        m = mass[0].cpu().numpy()
        see = visible(15 + r, 60, window, sinks)
        assert np.isfinite(m[~see]).all(), (r, np.flatnonzero(~np.isfinite(m) & ~see))
        assert np.isnan(m[see]).all(), r
    c.close()


@pytest.mark.parametrize("window,sinks", [(40, 3), (17, 0), (5, 21)])
@pytest.mark.parametrize("which", ["q", "K"])
def test_single_tokens_whose_weights_are_not_numbers_leave_other_keys_alone(which, window, sinks):
    """A query, or a key that it sees, is NaN: keys of the same blocks that the row does not see keep what they had."""
    c = Cache(2, 3, 64, [97, 300, 16], seed=24)
    c.batch(range(3), [1, 1, 1])
    mass = torch.full((3, 300), 0.25, device="cuda")
    if which == "q":
        c.qd[:] = float("nan")
    else:
        for i, n in enumerate(c.lens):
            c.K[0][i][n - 1] = np.nan
            c.write(0, i)
    for add in (True, False):
        c.attend(window=window, sinks=sinks, mass=mass, add=add)
        m = mass.cpu().numpy()
        for i, n in enumerate(c.lens):
            see = visible(n - 1, n, window, sinks)
            assert (m[i, :n][~see] == (0.25 if add else 0.0)).all(), (i, np.flatnonzero(m[i, :n] != 0.25))
            assert np.isnan(m[i, :n][see]).all() and (m[i, n:] == 0.25).all()
    c.close()


def test_weights_launch_what_there_is_to_sum():
    """A short prompt beside long single tokens, and a long one beside short ones: a
    tile of 128 keys a KV head and part for the prompts, 256 keys a workgroup for
    the single tokens, and nothing for the others' lengths."""
    def n_wgs(kv, group, lens, ql):
        tiles = sum(-(-n // 128) for n, q in zip(lens, ql) if q > 1)
        one = [n for n, q in zip(lens, ql) if q == 1]
        rows = -(-max(ql) // (32 // group))
        parts = min(16, max(1, 1024 // (tiles * kv)), rows)
        return tiles * kv * parts + tiles + len(one) * -(-max(one) // 256)

    for kv, group, lens, ql in [(4, 2, [100] + [3000 + 40 * i for i in range(24)], [20] + [1] * 24),
                                (2, 3, [5000, 130] + [60 + i for i in range(20)], [3, 40] + [1] * 20)]:
        c = Cache(kv, group, 128, lens, seed=25)
        c.batch(range(len(lens)), ql)
        mass = torch.zeros((len(lens), max(lens)), device="cuda")
        for window, sinks in [(0, 0), (90, 5)]:
            c.attend(window=window, sinks=sinks, mass=mass)
            check(c, window, sinks, mass=mass)
            assert c.eng.exec_counters()[6] == n_wgs(kv, group, lens, ql)
        c.close()


@pytest.mark.parametrize("kind", ["one item a row", "few rows of a long cache", "chunk"])
@pytest.mark.parametrize("scale", [2.0 ** 12, 2.0 ** 19, 2.0 ** 21, 2.0 ** 24])
def test_weights_of_large_scores_come_to_one_a_head(kind, scale):
    """Scores of four times the scale: from 2^23 on one rounding of a float32 score
    is a factor of 2 or more in a weight.  The weights are terms of the attention's
    own sums on every path: at most half an ulp of a score below 2^14 apart, 2^-11 in
    the exponent, ln 2 of that in the weight (3.4e-4)."""
    print(f"[gpu] large scores {kind} {scale}", flush=True)
    if kind == "few rows of a long cache":
        c = Cache(1, 1, 64, [16001, 15000, 16384, 16383], seed=26, scale=scale)
        c.batch(range(4), [2, 1, 1, 1])
    else:
        c = Cache(2, 4, 128, [200, 90, 1000], seed=27, scale=scale)
        if kind == "one item a row":
            c.eng.set_tuning(6, 0)
        c.batch([0, 1, 2], [40, 1, 30])
    heads = c.kv * c.group
    mass = torch.zeros((len(c.lens), max(c.lens)), device="cuda")
    for window, sinks in [(0, 0), (30, 2), (700, 40)]:
        c.attend(window=window, sinks=sinks, mass=mass)
        assert np.isfinite(c.out()).all()
        for i, ql in enumerate(c.q_lens):
            m = mass[i, :c.lens[i]].double().cpu().numpy()
            assert abs(m.sum() - ql * heads) < 5e-4 * ql * heads, (window, i, m.sum())
    c.close()
