"""The 4-bit calls on the CPU: sizes, refusals (nothing is launched for a bad
argument), and the format's reference against itself."""
import numpy as np
import pytest

import mx4_case as mx
from cache_case import model

vsk = pytest.importorskip("paper_2609_37062_amd.vsk")

A = 1 << 32  # aligned addresses that no refused call touches
B, W, Y, D = 2 * A, 3 * A, 4 * A, 5 * A


def _code(f, *a, **k):
    with pytest.raises(vsk.VskError) as x:
        f(*a, **k)
    return x.value.code


def test_reference_rounds_to_the_nearest_code():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((40, 96)) * 2.0 ** rng.integers(-20, 20, (40, 1))).astype(np.float32)
    v, e = mx.values(x), mx.exponents(x).astype(np.int64) - 127
    grid = np.concatenate([mx.GRID, -mx.GRID])
    for i in range(40):
        for b in range(3):
            g = np.ldexp(grid, e[i, b])
            err = np.abs(x[i, 32 * b:32 * b + 32, None] - g).min(axis=-1)
            np.testing.assert_array_equal(np.abs(v[i, 32 * b:32 * b + 32] - x[i, 32 * b:32 * b + 32]), err)
            top = np.abs(x[i, 32 * b:32 * b + 32]).max()
            assert 4 * 2.0 ** e[i, b] <= top < 8 * 2.0 ** e[i, b]
    # every tie and border of one block, both signs
    t = np.array([0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.9, 4.0] + [0.0] * 21)
    np.testing.assert_array_equal(mx.values(t)[:11], [0, 0, 1, 1, 2, 2, 4, 4, 6, 6, 4])
    np.testing.assert_array_equal(mx.values(-t), -mx.values(t))
    assert np.isnan(mx.values(np.array([1.0, np.inf]))).all() and mx.exponents(np.zeros(5))[0] == 0


def test_matrix_bytes():
    # 1 KiB a tile of 16 x 128, 256 bytes of exponents for four of them
    assert vsk.mx4_bytes(1, 1) == 1024 + 256
    assert vsk.mx4_bytes(16, 512) == 4 * 1024 + 256
    assert vsk.mx4_bytes(17, 513) == 2 * 5 * 1024 + 2 * 2 * 256
    assert vsk.mx4_product_bytes(17, 30, 513) >= vsk.mx4_bytes(17, 513)
    for bad in ((0, 5), (5, 0), (-1, 5), (5, -1), (1 << 30, 1 << 30), ((1 << 30) + 1, 1)):
        assert vsk.mx4_bytes(*bad) == 0
    assert vsk.mx4_product_bytes(4, 0, 5) == 0 and vsk.mx4_product_bytes(0, 4, 5) == 0


def test_matrix_refusals():
    q = lambda src=A, dtype=vsk.BF16, stride=100, rows=3, k=100, dst=B: vsk.mx4_quantise(src, dtype, stride, rows, k, dst)
    r = lambda src=A, rows=3, k=100, dst=B, dtype=vsk.BF16, stride=100: vsk.mx4_read(src, rows, k, dst, dtype, stride)
    p = lambda codes=A, scales=B, rows=3, k=100, dst=D: vsk.mx4_pack(codes, scales, rows, k, dst)
    for f, bads in (
        (q, (dict(src=None), dict(dst=None), dict(dtype=vsk.MX4), dict(dtype=-1), dict(stride=99), dict(rows=0), dict(k=0),
             dict(dst=B + 128), dict(src=A + 1), dict(src=A + 2, dtype=vsk.FP32), dict(dst=A), dict(src=B + 1024),
             dict(rows=1 << 30, k=1 << 30, stride=1 << 30), dict(stride=1 << 62))),
        (r, (dict(src=None), dict(dst=None), dict(dtype=vsk.MX4), dict(stride=99), dict(rows=-1), dict(src=A + 16),
             dict(dst=B + 1), dict(dst=B + 2, dtype=vsk.FP32), dict(dst=A + 1024), dict(stride=1 << 62))),
        (p, (dict(codes=None), dict(scales=None), dict(dst=None), dict(rows=0), dict(dst=D + 64), dict(codes=D), dict(scales=D)))):
        for bad in bads:
            assert _code(f, **bad) == "ARG", bad


def test_product_refusals():
    def f(x=A, xt=vsk.BF16, xs=256, w=W, rows=5, n=40, k=256, y=Y, yt=vsk.BF16, ys=40, ws=D, nbytes=1 << 20, add=None):
        vsk.mx4_product(x, xt, xs, w, rows, n, k, y, yt, ys, ws, nbytes, add_ptr=add)
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(xt=3), dict(yt=vsk.MX4), dict(xs=255), dict(ys=39), dict(rows=0),
                dict(n=0), dict(k=0), dict(x=A + 1), dict(x=A + 2, xt=vsk.FP32), dict(w=W + 128), dict(y=Y + 1),
                dict(y=Y + 2, yt=vsk.FP32), dict(ws=None), dict(ws=D + 16), dict(nbytes=vsk.mx4_product_bytes(5, 40, 256) - 1),
                dict(x=A + 16, xt=vsk.MX4), dict(y=A), dict(y=W + 64), dict(add=Y + 2), dict(add=Y + 1), dict(ws=A), dict(ws=W),
                dict(ws=Y), dict(add=D), dict(n=1 << 30, k=1 << 30), dict(xs=1 << 62), dict(ys=1 << 62)):
        assert _code(f, **bad) == "ARG", bad


def _engine(pool=None, four=True):
    e = vsk.Engine(model(2, 4, 64, 2, 512))
    e.kv_init(pool, 64)
    if four:
        e.kv4_init(A, e.kv4_pool_bytes(64))
    for i, n in enumerate((100, 40, 17)):
        e.seq_create(i)
        e.reserve(i, n)
    return e


def test_cache_bytes_and_binding():
    e = vsk.Engine(model(2, 4, 64, 3, 512))
    assert e.kv4_pool_bytes(10) == 3 * 10 * 2 * 17 * 64
    assert e.kv4_pool_bytes(10) * 64 == e.kv_pool_bytes(10) * 17
    assert e.kv4_pool_bytes(0) == 0
    assert _code(e.kv4_init, A, 1 << 30) == "STATE"  # before kv_init
    e.kv_init(None, 10)
    assert _code(e.kv4_init, A, e.kv4_pool_bytes(10) - 1) == "ARG"
    assert _code(e.kv4_init, A + 64, 1 << 30) == "ARG"
    assert _code(e.kv4_write, 0, B, 1, W, Y) == "STATE"
    e.kv4_init(A, e.kv4_pool_bytes(10))
    e.kv4_init(None)
    assert _code(e.kv4_read, 0, B, 1, W, Y) == "STATE"
    e.kv4_init(A, e.kv4_pool_bytes(10))
    e.kv_init(None, 20)  # another pool size: bound again
    assert _code(e.kv4_read, 0, B, 1, W, Y) == "STATE"
    assert e.rope_bytes() == 512 * 32 * 24
    e.close()


def test_cache_refusals():
    e = _engine()
    for f in (e.kv4_write, e.kv4_read):
        for bad, code in (((2, B, 1, W, Y), "RANGE"), ((-1, B, 1, W, Y), "RANGE"), ((0, B, -1, W, Y), "ARG"), ((0, None, 1, W, Y), "ARG"),
                          ((0, B, 1, None, Y), "ARG"), ((0, B, 1, W, None), "ARG"), ((0, B + 2, 1, W, Y), "ARG"),
                          ((0, B, 1, W + 1, Y), "ARG"), ((0, B, 1, W, Y + 1), "ARG")):
            assert _code(f, *bad) == code, bad
    assert _code(e.kv4_attend, 0, B, W, Y, 256) == "STATE"  # no batch
    assert _code(e.qkv_norm_rope, 0, B, 768, None, None, W, 4) == "STATE"  # no rotary table
    assert _code(e.qkv_norm_rope, 0, B, 768, None, None, W, 16) == "STATE"  # no 16-bit pool
    assert _code(e.qkv_norm_rope, 0, B, 768, None, None, W, 8) == "ARG"
    assert _code(e.rope_bind, None, 1 << 30) == "ARG"
    assert _code(e.rope_bind, B + 8, 1 << 30) == "ARG"
    assert _code(e.rope_bind, B, e.rope_bytes() - 1) == "ARG"
    e.close()
    e = _engine(four=False)
    assert _code(e.kv4_attend, 0, B, W, Y, 256) == "STATE"
    assert _code(e.qkv_norm_rope, 0, B, 768, None, None, W, 4) == "STATE"
    e.close()


def test_eviction_refuses_a_four_bit_cache():
    e = _engine(pool=B)
    e.seq_create(7)
    free = e.free_blocks()
    assert _code(e.kv_evict, [7], [0], [20], 2, 4, W, 100, Y, 1 << 16, kept_ptr=D, out_stride=32) == "UNSUPPORTED"
    assert e.free_blocks() == free
    e.close()


def test_sizes_that_no_launch_takes_are_refused():
    """A wave a tile, eight values of a head a thread, less than 2^32 threads a launch."""
    most = (1 << 26) - 4
    assert vsk.mx4_bytes(16 * most, 1) == most * (1024 + 256)
    assert vsk.mx4_bytes(1, 1 << 30) == (1 << 23) * 1024 + (1 << 21) * 256
    for rows, k in ((16 * most + 1, 1), (1 << 30, 1), (8192 * 16, 8192 * 128)):
        assert vsk.mx4_bytes(rows, k) == 0, (rows, k)
        assert _code(vsk.mx4_read, A, rows, k, 1 << 50, vsk.BF16, k) == "ARG"
        assert _code(vsk.mx4_pack, A, B, rows, k, 1 << 50) == "ARG"
        assert vsk.mx4_product_bytes(rows, 5, k) == 0 and vsk.mx4_product_bytes(5, rows, k) == 0
    e = _engine()
    for f in (e.kv4_write, e.kv4_read):
        for n in ((1 << 28) - 8, (1 << 31) - 1):
            assert _code(f, 0, B, n, W, Y) == "ARG", n
    e.close()
