"""The 4-bit operators one after the other, as a layer of a served model uses them: a
product to queries, keys and values, their norms and rotation into the 4-bit cache,
attention over it, and a product back into the residual stream."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import mx4_case as mx  # noqa: E402
from cache_case import U  # noqa: E402
from mx4_case import Cache4, check_rows, turned  # noqa: E402

pytestmark = pytest.mark.gpu

EPS, THETA = float(np.float32(1e-5)), 500000.0


class Layer:
    """Weights of one attention layer beside a Cache4, and a residual stream."""

    def __init__(self, c, hidden, seed):
        from paper_2609_37062_amd import vsk
        self.c, self.vsk, self.hidden = c, vsk, hidden
        rng = np.random.default_rng(seed)
        self.width, self.nq = c.kv * (c.group + 2) * c.hd, c.kv * c.group * c.hd
        self.w, self.mx = [], []
        for n, k in ((self.width, hidden), (hidden, self.nq)):
            w = rng.standard_normal((n, k)) * 2.0 / np.sqrt(k)
            self.w.append(mx.values(w))
            codes = torch.from_numpy(mx.in_file(mx.codes(w))).cuda()
            exps = torch.from_numpy(mx.exponents(w)).cuda()
            t, at = c.buf(vsk.mx4_bytes(n, k), "cuda")
            vsk.mx4_pack(codes.data_ptr(), exps.data_ptr(), n, k, at, c.sp)
            torch.cuda.synchronize()
            self.mx.append((t, at))
        self.gains = torch.from_numpy(1 + 0.3 * rng.standard_normal((2, c.hd))).to(torch.bfloat16).cuda()
        nb = c.eng.rope_bytes()
        self.rope, at = c.buf(nb, "cuda")
        c.eng.rope_bind(at, nb, c.sp)

    def batch(self, seqs, q_lens, seed):
        """A batch and its buffers."""
        c, rows = self.c, sum(q_lens)
        c.batch(seqs, q_lens)
        rng = np.random.default_rng(seed)
        self.rows = rows
        self.h = torch.from_numpy(rng.standard_normal((rows, self.hidden)).astype(np.float32)).cuda()
        self.x = torch.zeros((rows, self.hidden), dtype=torch.bfloat16, device="cuda")
        self.qkv = torch.zeros((rows, self.width), dtype=torch.bfloat16, device="cuda")
        self.y = torch.zeros_like(self.h)
        self.ws = self.workspace()

    def workspace(self):
        """Scratch for both products, one after the other."""
        v = self.vsk
        nb = max(v.mx4_product_bytes(self.rows, self.width, self.hidden), v.mx4_product_bytes(self.rows, self.hidden, self.nq))
        t, at = self.c.buf(nb, "cuda")
        t.fill_(-1)
        return t, at, nb

    def run(self, stream, layer=0, window=0, sinks=0):
        c, v, R = self.c, self.vsk, self.rows
        _, ws, nb = self.ws
        self.x.copy_(self.h * torch.rsqrt((self.h * self.h).mean(dim=-1, keepdim=True) + 1e-5))
        v.mx4_product(self.x.data_ptr(), v.BF16, self.hidden, self.mx[0][1], R, self.width, self.hidden, self.qkv.data_ptr(),
                      v.BF16, self.width, ws, nb, stream=stream)
        c.eng.qkv_norm_rope(layer, self.qkv.data_ptr(), self.width, self.gains[0].data_ptr(), self.gains[1].data_ptr(),
                            c.qd.data_ptr(), 4, stream)
        c.attend(layer, window, sinks, stream=stream)
        v.mx4_product(c.o.data_ptr(), v.BF16, self.nq, self.mx[1][1], R, self.hidden, self.nq, self.y.data_ptr(), v.FP32,
                      self.hidden, ws, nb, add_ptr=self.h.data_ptr(), stream=stream)

    def check(self, layer=0, window=0, sinks=0):
        """Each call's output against 64 bits, from the device's own inputs to that call."""
        c = self.c
        torch.cuda.synchronize()
        f64 = lambda t: t.float().cpu().numpy().astype(np.float64)
        xv, qkv = mx.values(f64(self.x)), f64(self.qkv)
        want, mag = xv @ self.w[0].T, np.abs(xv) @ np.abs(self.w[0]).T
        assert (np.abs(qkv - want) <= self._sums(self.hidden) * mag * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)).all()
        b = c.eng.batch_host()
        pos, g = b["pos"].astype(np.float64), f64(self.gains)
        rows = qkv.reshape(self.rows, -1, c.hd)
        heads = c.kv * c.group
        q, mq = turned(rows[:, :heads], pos, g[0], THETA, EPS)
        k, _ = turned(rows[:, heads:heads + c.kv], pos, g[1], THETA, EPS)
        # (40 half steps of float32 and one of bf16, as counted where the rows are tested alone)
        assert (np.abs(f64(c.qd).reshape(q.shape) - q) <= 40 * U * mq + 2.0 ** -8 * np.abs(q) + 1e-38).all()
        r0 = 0
        for s, ql in zip(c.seqs, c.q_lens):
            c.K[layer][s][-ql:] = mx.values(k[r0:r0 + ql])
            c.V[layer][s][-ql:] = mx.values(rows[r0:r0 + ql, heads + c.kv:])
            K, V = c.read(layer, s)
            np.testing.assert_array_equal(K, c.K[layer][s])
            np.testing.assert_array_equal(V, c.V[layer][s])
            r0 += ql
        c.q = c.qd.reshape(c.q.shape).cpu()
        check_rows(c, window, sinks, layer)
        o = mx.values(f64(c.o[:-1]).reshape(self.rows, -1))
        h = f64(self.h)
        want, mag = o @ self.w[1].T + h, np.abs(o) @ np.abs(self.w[1]).T + np.abs(h)
        assert (np.abs(f64(self.y) - want) <= self._sums(self.nq) * mag).all()

    @staticmethod
    def _sums(k):
        """Products are exact; a sum of 128 of them and what is there already is off by at
        most two steps of float32 of the magnitudes in it, a join of partial sums and the
        addend by one each (16 of them at most)."""
        return (4 * ((k + 127) // 128) + 2 * 16) * U


CONFIGS = [(2, 4, 128, 640), (1, 3, 64, 200), (4, 1, 64, 256)]


@pytest.mark.parametrize("kv,group,hd,hidden", CONFIGS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 4)])
def test_a_layer(kv, group, hd, hidden, window, sinks):
    """Prompt rows and single tokens, then a decode step, in both layers of a cache."""
    print(f"[gpu] layer of 4 bits kv={kv} group={group} hd={hd} window={window}", flush=True)
    c = Cache4(kv, group, hd, [1, 200, 37, 333, 90], layers=2, seed=hidden + window)
    layer = Layer(c, hidden, seed=kv)
    for i, (seqs, q_lens) in enumerate((([0, 1, 2, 3, 4], [1, 60, 37, 1, 18]), ([0, 1, 2, 3, 4], [1] * 5), ([3], [1]), ([3, 1], [300, 5]))):
        layer.batch(seqs, q_lens, seed=i)
        for n in range(2):
            layer.run(c.sp, n, window, sinks)
            layer.check(n, window, sinks)
    c.close()


def test_layers_captured_share_workspaces():
    """Two layers as two graphs over the same workspaces, replayed in turn with eager
    calls between them: every replay is the eager call, bit by bit."""
    c = Cache4(2, 4, 128, [400, 90, 1000], layers=2, seed=3)
    layer = Layer(c, 512, seed=4)
    layer.batch([0, 1, 2], [45, 1, 1], seed=5)
    spans = ((0, 0), (64, 4))
    graphs = []
    for n in range(2):
        layer.run(c.sp, n, *spans[n])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            layer.run(torch.cuda.current_stream().cuda_stream, n, *spans[n])
        graphs.append(g)
    for i in range(3):
        layer.h.copy_(torch.randn_like(layer.h))
        for n in (0, 1):
            outs = []
            for call in (graphs[n].replay, lambda: layer.run(c.sp, n, *spans[n])):
                layer.y.zero_()
                c.o[:-1].zero_()
                call()
                outs.append((layer.y.clone(), c.o.clone(), layer.qkv.clone(), c.qd.clone()))
            torch.cuda.synchronize()
            for a, b in zip(*outs):
                assert torch.equal(a, b), (i, n)
            layer.check(n, *spans[n])
    c.close()


def test_two_layers_at_once():
    """Two handles on two streams, each with workspaces of its own: as one after the other."""
    layers = []
    for i in range(2):
        c = Cache4(2, 4, 128, [700, 90 + i, 300], seed=20 + i)
        layers.append(Layer(c, 512, seed=i))
        layers[i].batch([0, 1, 2], [100, 1, 40], seed=i)
    want = []
    for layer in layers:
        layer.run(layer.c.sp)
        layer.check()
        want.append((layer.y.clone(), layer.c.o.clone()))
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(3):
        for layer in layers:
            layer.y.zero_()
        torch.cuda.synchronize()
        for layer, s in zip(layers, streams):
            with torch.cuda.stream(s):
                for _ in range(4):
                    layer.run(s.cuda_stream)
        torch.cuda.synchronize()
        for layer, (y, o) in zip(layers, want):
            assert torch.equal(layer.y, y) and torch.equal(layer.c.o, o)
    for layer in layers:
        layer.c.close()


def test_both_caches_side_by_side():
    """The 16-bit and the 4-bit pool of one handle: either is written and read alone."""
    c = Cache4(2, 2, 64, [70, 33], seed=9)
    layer = Layer(c, 128, seed=9)
    layer.batch([0, 1], [20, 33], seed=1)
    torch.cuda.synchronize()
    before4, before = c._pool4.clone(), c.pool.clone()
    layer.run(c.sp)
    torch.cuda.synchronize()
    assert torch.equal(c.pool, before) and not torch.equal(c._pool4, before4)
    before4 = c._pool4.clone()
    c.eng.qkv_norm_rope(0, layer.qkv.data_ptr(), layer.width, layer.gains[0].data_ptr(), layer.gains[1].data_ptr(),
                        c.qd.data_ptr(), 16, c.sp)
    torch.cuda.synchronize()
    assert torch.equal(c._pool4, before4) and not torch.equal(c.pool, before)
    layer.check()
    # a new 16-bit pool forgets the sequences and unbinds the 4-bit one
    c.eng.kv_init(c.pool.data_ptr(), c.n_blocks)
    with pytest.raises(layer.vsk.VskError) as e:
        c.eng.kv4_write(0, c.qd.data_ptr(), 1, c.qd.data_ptr(), c.qd.data_ptr(), c.sp)
    assert e.value.code == "STATE"
    c.close()
