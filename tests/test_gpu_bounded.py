"""Passes over bounded caches: layers with a window and sinks, the weights per token
that passes leave, and passes over evicted sequences, against the float64
oracle; and the whole of it as a server runs it, a prompt, evictions and steps.

The oracle's attention is replaced by one that applies the window and keeps the
weights; everything else of the pass is the oracle's own."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from helpers import compare_logits, e2e_compare  # noqa: E402
from oracle import numerics as nm  # noqa: E402
from oracle.kvcache import PagedKV  # noqa: E402
from oracle.model import GeneratedWeights, forward  # noqa: E402
from workloads.configs import ModelCfg, decode_workload, mixed_workload  # noqa: E402

pytestmark = pytest.mark.gpu

MID = ModelCfg("bounded-2L", n_layers=2, hidden=512, n_q_heads=8, n_kv_heads=2, head_dim=128, ffn=1024, vocab=1024)

# A pass's q and new K come out of bf16 roundings that may differ from the
# oracle's in a tenth of the elements by a step (2^-7): a score of d = 128
# terms of unit size is then off by 2 * 0.1 * 2^-7 * 7.2 at most, and a weight
# by twice that.
MASS_TOL = 0.03


class Spanned:
    """The oracle's attend with the spans of the layers; keeps every weight row."""

    def __init__(self, spans, calls_per_layer):
        self.spans, self.per, self.n, self.rows = spans, calls_per_layer, 0, []

    def __call__(self, q, K, V, dt=np.float64):
        window, sinks = self.spans[self.n // self.per % len(self.spans)]
        self.n += 1
        n = len(K)
        t = np.arange(n)
        see = (t > n - 1 - window) | (t < sinks) if window else t >= 0
        q = np.asarray(q, dt)
        s = (np.asarray(K[see], dt) @ q) / dt(np.sqrt(q.shape[-1]))
        p = np.exp(s - np.max(s))
        p /= np.sum(p, dtype=dt)
        full = np.zeros(n)
        full[see] = p
        self.rows.append(full)
        return p @ np.asarray(V[see], dt)


def _run(w, **kw):
    from paper_2609_37062_amd.runner import DeviceRun
    print(f"[gpu] bounded: {w.name} rows={w.n_rows}", flush=True)
    return DeviceRun(w, poison_pool=True, **kw)


@pytest.mark.parametrize("spans", [[(20, 4), (0, 0)], [(0, 0), (1, 0)], [(300, 17), (33, 40)]])
@pytest.mark.parametrize("kind", ["decode", "mixed"])
def test_passes_with_windows(spans, kind, monkeypatch):
    if kind == "decode":
        w = decode_workload(MID, [0, 15, 16, 40, 333, 700], seed=21, name="window-decode")
    else:
        w = mixed_workload(MID, 2, 61, [0, 50, 400], seed=22, name="window-mixed")
    d = _run(w)
    for l, (window, sinks) in enumerate(spans):
        d.eng.set_span(l, window, sinks)
    d.step()
    lg, ids = d.results()
    monkeypatch.setattr(nm, "attend", Spanned(spans, w.n_rows * MID.n_q_heads))
    e2e_compare(w, lg, ids)
    d.release()


def test_a_window_over_everything_changes_no_bit():
    w = decode_workload(MID, [5, 90, 333], seed=23, name="window-all")
    d = _run(w)
    d.step()
    a = d.results()
    d.eng.set_span(-1, MID.max_pos, 3)
    d.step()
    b = d.results()
    d.eng.set_span(-1, 7, 3)
    d.step()
    c = d.results()
    d.eng.set_span(-1, 0)
    d.step()
    e = d.results()
    np.testing.assert_array_equal(a[0], b[0])
    np.testing.assert_array_equal(a[0], e[0])
    assert (a[0] != c[0]).any()
    d.eng.set_span(1, 7, 3)
    d.eng.set_tuning(2, 2)
    with pytest.raises(Exception) as x:
        d.step()
    assert x.value.code == "UNSUPPORTED"
    d.release()


@pytest.mark.parametrize("spans", [[(0, 0), (0, 0)], [(30, 4), (0, 0)]])
def test_passes_leave_weights(spans, monkeypatch):
    w = mixed_workload(MID, 2, 37, [3, 50, 200], seed=24, name="mass-mixed")
    d = _run(w)
    for l, (window, sinks) in enumerate(spans):
        d.eng.set_span(l, window, sinks)
    kvmax = max(s.ctx + s.q_len for s in w.seqs)
    d.step()
    plain = d.results()[0]
    mass = torch.zeros((w.n_seqs + 1, kvmax + 5), device="cuda")
    mass[:, :] = 2.0
    d.eng.set_mass(mass.data_ptr(), w.n_seqs + 1, kvmax + 5)
    d.step()
    lg, ids = d.results()
    att = Spanned(spans, w.n_rows * MID.n_q_heads)
    monkeypatch.setattr(nm, "attend", att)
    e2e_compare(w, lg, ids)
    assert np.abs(lg - plain).max() < 0.05  # (another walk, the same pass)
    m = mass.cpu().numpy().astype(np.float64)
    at = 0
    want = [np.zeros(s.ctx + s.q_len) for s in w.seqs]
    for _ in range(MID.n_layers):  # (the float64 run's rows come first)
        for i, s in enumerate(w.seqs):
            for _ in range(s.q_len * MID.n_q_heads):
                row = att.rows[at]
                want[i][:len(row)] += row
                at += 1
    for i, x in enumerate(want):
        assert (m[i, len(x):] == 2.0).all()
        np.testing.assert_allclose(m[i, :len(x)] - 2.0, x, rtol=MASS_TOL, atol=1e-5)
    assert (m[-1] == 2.0).all()
    # room for too few sequences or too short ones: refused
    for n, stride in ((w.n_seqs - 1, kvmax), (w.n_seqs, kvmax - 1)):
        d.eng.set_mass(mass.data_ptr(), n, stride)
        with pytest.raises(Exception) as x:
            d.step()
        assert x.value.code == "ARG"
    d.eng.set_mass(None)
    before = mass.clone()
    d.step()
    torch.cuda.synchronize()
    assert torch.equal(before, mass)
    d.release()


def test_project_only_rows_leave_no_weights():
    w = mixed_workload(MID, 2, 21, [60, 33, 5], seed=25, name="mass-routed")
    d = _run(w, routed=True)
    rng = np.random.default_rng(1)
    L, R = MID.n_routed, w.n_rows
    run = rng.random((L, R)) < 0.5
    d.set_route(run, np.ones((L, R), np.float32))
    mass = torch.zeros((w.n_seqs, 100), device="cuda")
    for spans in ((0, 0), (9, 2)):
        d.eng.set_span(-1, *spans)
        mass.zero_()
        d.eng.set_mass(mass.data_ptr(), w.n_seqs, 100)
        d.step_routed()
        d.results()
        m = mass.cpu().numpy()
        r0 = 0
        for i, s in enumerate(w.seqs):
            n = run[:, r0:r0 + s.q_len].sum() + (MID.n_layers - L) * s.q_len
            np.testing.assert_allclose(m[i].sum(), n * MID.n_q_heads, rtol=1e-4)
            r0 += s.q_len
    d.release()


def _oracle_of(d, seqs, spans=None):
    """The oracle's state of the device's cache and batch."""
    m = d.m
    b = d.eng.batch_host()
    kv = PagedKV(m.n_layers, d.n_blocks, m.n_kv_heads, m.head_dim)
    for s in seqs:
        n, _ = d.eng.seq_info(s)
        sl = d.seq_slots(s, 0, n)
        for l in range(m.n_layers):
            K, V = d.read_kv(l, sl)
            kv.write(l, sl, np.nan_to_num(K), np.nan_to_num(V))  # (the new rows' slots hold nothing yet)
    return b, kv


def _checked_step(d, w, seqs, tokens, layers_spans, monkeypatch):
    """One decode step of the listed sequences against the oracle; returns its ids."""
    for s in seqs:
        d.eng.reserve(s, 1)
    d.rebatch(seqs)
    d.ids = torch.from_numpy(np.ascontiguousarray(tokens, np.int32)).cuda()
    b, kv = _oracle_of(d, seqs)
    d.step()
    lg, ids = d.results()
    W = GeneratedWeights(d.m, w.seed, cache=True)
    per = len(seqs) * d.m.n_q_heads
    z = {}
    for dt in ("f64", "f32"):
        monkeypatch.setattr(nm, "attend", Spanned(layers_spans, per))
        z[dt] = forward(d.m, W, kv, b, tokens, np.arange(len(seqs)), dtype=dt)["z"]
    compare_logits(lg[:len(seqs)], ids[:len(seqs)], z["f64"], z32=z["f32"])
    return ids[:len(seqs)]


@pytest.mark.parametrize("spans", [[(0, 0), (0, 0)], [(25, 4), (0, 0)]])
def test_a_conversation_in_a_bounded_cache(spans, monkeypatch):
    """Prompts that leave their weights, eviction, steps that go on counting,
    another eviction, more steps: every step's logits against the oracle run on
    the tokens that are still there, at their own positions."""
    from paper_2609_37062_amd.runner import _dev_buffer
    w = mixed_workload(MID, 2, 90, [120], seed=26, name="conversation")
    d = _run(w, pool_blocks=200, max_kv_len=256)
    for l, (window, sinks) in enumerate(spans):
        d.eng.set_span(l, window, sinks)
    n = w.n_seqs
    mass = torch.zeros((n, 256), device="cuda")
    d.eng.set_mass(mass.data_ptr(), n, 256)
    d.step()
    _, ids = d.results()
    tokens = np.asarray(ids[:n], np.int32)
    seqs = list(range(n))
    drop = 0
    for cut in (40, 38):
        lens = [d.eng.seq_info(s)[0] for s in seqs]
        keep = [min(cut, x) for x in lens]
        dst = [s + 100 for s in seqs]
        for s in dst:
            d.eng.seq_create(s)
        kept = torch.empty((n, 256), dtype=torch.int32, device="cuda")
        nb = d.eng.kv_evict_bytes(seqs, keep)
        t, meta = _dev_buffer(nb, "cuda")
        before = mass.cpu().numpy()
        d.eng.kv_evict(dst, seqs, keep, 4, 16, mass.data_ptr(), 256, meta, nb, mass_out_ptr=mass.data_ptr(),
                       kept_ptr=kept.data_ptr(), out_stride=256, stream=d.sp)
        for s in seqs:
            d.eng.seq_release(s)
        torch.cuda.synchronize()
        for i, (k, ln) in enumerate(zip(keep, lens)):
            x = kept[i, :k].cpu().numpy()
            assert (np.diff(x) > 0).all() and x[0] == 0 and x[-1] == ln - 1
            rest = np.setdiff1d(np.arange(ln), x)
            assert len(rest) == 0 or before[i, x[4:-16]].min() >= before[i, rest].max()
        seqs = dst
        for _ in range(2):
            tokens = np.asarray(_checked_step(d, w, seqs, tokens, spans, monkeypatch), np.int32)
            drop += 1
    torch.cuda.synchronize()
    m = mass.cpu().numpy()
    for i, s in enumerate(seqs):
        ln = d.eng.seq_info(s)[0]
        assert ln == 40 and (m[i, ln:] == 0).all() and (m[i, :ln] > 0).any()
    # positions never went back: the tokens seen so far
    b = d.eng.batch_host()
    np.testing.assert_array_equal(b["pos"], [sp.ctx + sp.q_len + drop - 1 for sp in w.seqs])
    d.release()


@pytest.mark.parametrize("kind", ["decode", "mixed"])
def test_replayed_passes_add_weights(kind):
    """A captured pass over a windowed layer and a full one: every replay, with eager
    passes between, gives the eager pass's bits and adds the same weights."""
    if kind == "decode":
        w = decode_workload(MID, [7, 16, 90, 500], seed=27, name="replay-decode")
    else:
        w = mixed_workload(MID, 1, 45, [3, 300], seed=28, name="replay-mixed")
    d = _run(w)
    n = max(s.ctx + s.q_len for s in w.seqs)
    mass = torch.zeros((w.n_seqs, n), device="cuda")
    d.eng.set_span(0, 30, 4)
    d.eng.set_mass(mass.data_ptr(), w.n_seqs, n)
    d.step()
    lg, ids = d.results()
    once = mass.clone()
    assert float(once.sum()) > 0
    d.step()
    torch.cuda.synchronize()
    twice = mass.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        d.step(torch.cuda.current_stream().cuda_stream)
    for _ in range(4):
        mass.zero_()
        d.logits.zero_()
        g.replay()
        a, b = d.results()
        np.testing.assert_array_equal(a, lg)
        np.testing.assert_array_equal(b, ids)
        assert torch.equal(mass, once)
        d.step()
        torch.cuda.synchronize()
        assert torch.equal(mass, twice)
    d.release()


def test_the_scratch_entry_sees_windows_and_leaves_weights():
    w = decode_workload(MID, [7, 16, 90, 500], seed=27, name="scratch-decode")
    d = _run(w)
    mass = torch.zeros((2, 4, 501), device="cuda")
    d.eng.set_span(1, 30, 4)
    d.eng.set_mass(mass[0].data_ptr(), 4, 501)
    d.step()
    a = d.results()
    d.logits.zero_()
    d.eng.set_mass(mass[1].data_ptr(), 4, 501)
    d.eng.decode_step_scratch(d.ids.data_ptr(), d.logits.data_ptr(), d.next_ids.data_ptr(), d.sp)
    b = d.results()
    np.testing.assert_array_equal(a[0], b[0])
    np.testing.assert_array_equal(a[1], b[1])
    assert torch.equal(mass[0], mass[1]) and float(mass[0].sum()) > 0
    d.eng.set_mass(mass[1].data_ptr(), 3, 501)
    with pytest.raises(Exception) as x:
        d.eng.decode_step_scratch(d.ids.data_ptr(), d.logits.data_ptr(), d.next_ids.data_ptr(), d.sp)
    assert x.value.code == "ARG"
    d.release()


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("kind", ["chunk", "one item a row", "prefix"])
def test_project_only_rows_leave_no_weights_on_keys_that_are_not_finite(kind, bad):
    """A layer whose rows are all Project-Only reads no K and V: what these hold changes no bit."""
    import dataclasses
    from workloads.configs import SeqSpec, prefix_groups_workload
    if kind == "prefix":
        w = prefix_groups_workload(MID, [(96, 3)], [10, 21, 5, 40], seed=29, name="po-prefix")
    else:
        w = mixed_workload(MID, 1, 19, [60, 33, 5], seed=30, name="po-chunk")
        s = w.seqs[1]
        seqs = [w.seqs[0], SeqSpec(60, 21, s.blocks, s.content, logits=True)] + w.seqs[2:]
        tokens = np.random.default_rng(31).integers(0, MID.vocab, 19 + 21 + 2).astype(np.int32)
        w = dataclasses.replace(w, seqs=seqs, tokens=tokens, n_pool_blocks=w.n_pool_blocks + 4)
    d = _run(w, routed=True)
    assert MID.n_routed == 1
    if kind == "one item a row":
        d.eng.set_tuning(6, 0)
    d.set_route(np.zeros((1, w.n_rows), bool), np.ones((1, w.n_rows), np.float32))
    n = max(s.ctx + s.q_len for s in w.seqs)
    mass = torch.zeros((w.n_seqs, n), device="cuda")
    d.eng.set_mass(mass.data_ptr(), w.n_seqs, n)
    want = {}
    for spans in ((0, 0), (40, 2)):
        d.eng.set_span(-1, *spans)
        mass.zero_()
        d.step_routed()
        want[spans] = (d.results()[0], mass.clone())
        assert float(mass.sum()) > 0
    for i, s in enumerate(w.seqs):
        if s.ctx:
            sl = torch.from_numpy(d.seq_slots(i, 0, s.ctx)).cuda()
            x = torch.full((s.ctx, MID.n_kv_heads, MID.head_dim), bad, dtype=torch.bfloat16, device="cuda")
            d.eng.kv_write(1, sl.data_ptr(), s.ctx, x.data_ptr(), x.data_ptr(), d.sp)
            torch.cuda.synchronize()
    for spans, (lg, m) in want.items():
        d.eng.set_span(-1, *spans)
        mass.zero_()
        d.step_routed()
        np.testing.assert_array_equal(d.results()[0], lg)
        assert torch.equal(mass, m), (spans, torch.nonzero(mass != m)[:5].tolist())
    d.release()


@pytest.mark.parametrize("window", [0, 9])
def test_probes_of_decode_attention_wait_for_a_decode_kernel(window):
    """A pass of prompt rows alone launches no decode attention: the next decode pass takes the pairs."""
    from bench import HipEvents
    w = mixed_workload(MID, 1, 33, [], seed=32, name="probe-prompt")
    d = _run(w, pool_blocks=8, max_kv_len=64)
    d.eng.set_span(-1, window, 0)
    ev = HipEvents()
    b, e = ev.create(3), ev.create(3)
    d.eng.set_probe(4, b, e)
    d.step()
    d.eng.reserve(0, 1)
    d.rebatch([0])
    d.step()
    torch.cuda.synchronize()
    for l in range(MID.n_layers):
        assert 0 < ev.elapsed_ms(b[l], e[l]) < 1000
    d.eng.set_probe(4, [], [])
    ev.destroy(b + e)
    d.release()


@pytest.mark.parametrize("kind", ["decode", "mixed"])
def test_alternating_windows_are_planned_once_each(kind, monkeypatch):
    import dataclasses
    m = dataclasses.replace(MID, name="bounded-5L", n_layers=5)
    spans = [(30, 4), (0, 0), (30, 4), (0, 0), (100, 4)]
    if kind == "decode":
        w = decode_workload(m, [3, 40, 333], seed=33, name="alternate-decode")
    else:
        w = mixed_workload(m, 1, 70, [5, 200], seed=34, name="alternate-mixed")
    d = _run(w)
    for l, (window, sinks) in enumerate(spans):
        d.eng.set_span(l, window, sinks)
    d.step()
    lg, ids = d.results()
    assert d.eng.exec_counters()[7] == 3
    monkeypatch.setattr(nm, "attend", Spanned(spans, w.n_rows * m.n_q_heads))
    e2e_compare(w, lg, ids)
    d.eng.set_span(-1, 30, 4)
    d.step()
    d.results()
    assert d.eng.exec_counters()[7] == 1
    d.release()
