"""Refusals of the bounded-cache calls, on the CPU: nothing is launched for a bad
argument, and the host allocator is left as it was."""
import numpy as np
import pytest

from cache_case import model

vsk = pytest.importorskip("paper_2609_37062_amd.vsk")

FAKE = 1 << 20  # an aligned address that no refused call touches


def _engine(pool=FAKE, layers=2, max_pos=512):
    e = vsk.Engine(model(2, 4, 64, layers, max_pos))
    e.kv_init(pool, 64)
    for i, n in enumerate((100, 40, 17)):
        e.seq_create(i)
        e.reserve(i, n)
    return e


def _code(f, *a, **k):
    with pytest.raises(vsk.VskError) as x:
        f(*a, **k)
    return x.value.code


def test_attend_refuses_before_a_batch_is_there():
    e = _engine(pool=None)
    assert _code(e.attend, 0, FAKE, 2 * FAKE, FAKE, 256) == "STATE"  # no pool
    e.close()
    e = _engine()
    assert _code(e.attend, 0, FAKE, 2 * FAKE, FAKE, 256) == "STATE"  # no batch uploaded
    e.batch_build([0], [1])
    assert _code(e.attend, 0, FAKE, 2 * FAKE, FAKE, 256) == "STATE"
    e.close()


def test_span_refusals():
    e = _engine()
    assert _code(e.set_span, 2, 4) == "RANGE"
    assert _code(e.set_span, -2, 4) == "RANGE"
    assert _code(e.set_span, 0, -1) == "ARG"
    assert _code(e.set_span, 0, 4, -1) == "ARG"
    e.set_span(0, 4, 2)
    e.set_span(-1, 0, 0)
    e.close()


def test_mass_refusals():
    e = _engine()
    assert _code(e.set_mass, FAKE, 0, 4) == "ARG"
    assert _code(e.set_mass, FAKE, 4, 0) == "ARG"
    assert _code(e.set_mass, FAKE + 2, 4, 4) == "ARG"
    e.set_mass(FAKE, 4, 4)
    e.set_mass(None)
    e.close()


def _evict(e, dst=(7,), src=(0,), keep=(20,), sinks=2, recent=4, mass=FAKE, stride=100, meta=8 * FAKE, nbytes=1 << 16,
           mass_out=None, kept=2 * FAKE, slots=None, out_stride=32):
    e.kv_evict(list(dst), list(src), list(keep), sinks, recent, mass, stride, meta, nbytes, mass_out_ptr=mass_out,
               kept_ptr=kept, slots_ptr=slots, out_stride=out_stride)


def test_evict_refusals():
    e = _engine()
    e.seq_create(7)
    e.seq_create(8)
    free = e.free_blocks()
    for bad, code in [
        (dict(dst=(), src=(), keep=()), "ARG"),
        (dict(dst=(7, 7), src=(0, 0), keep=(20, 20)), "ARG"), (dict(src=(5,)), "STATE"), (dict(dst=(9,)), "STATE"), (dict(dst=(1,)), "STATE"), (dict(dst=(0,)), "STATE"),
        (dict(keep=(0,)), "ARG"), (dict(keep=(101,)), "ARG"), (dict(keep=(-3,)), "ARG"),
        (dict(sinks=-1), "ARG"), (dict(recent=-1), "ARG"), (dict(sinks=17, recent=4), "ARG"),
        (dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), "ARG"),
        (dict(stride=99), "ARG"), (dict(out_stride=19), "ARG"),
        (dict(mass=None), "ARG"), (dict(kept=None), "ARG"), (dict(meta=None), "ARG"),
        (dict(mass=FAKE + 1), "ARG"), (dict(kept=FAKE * 2 + 2), "ARG"), (dict(meta=8 * FAKE + 16), "ARG"),
        (dict(nbytes=16), "ARG"),
        (dict(kept=FAKE), "ARG"), (dict(kept=FAKE + 396), "ARG"), (dict(slots=2 * FAKE), "ARG"),
        (dict(slots=FAKE + 8), "ARG"), (dict(mass_out=FAKE + 4), "ARG"), (dict(mass_out=FAKE), "ARG"),
        (dict(mass_out=2 * FAKE), "ARG"), (dict(mass_out=3 * FAKE, slots=3 * FAKE + 64), "ARG"),
    ]:
        assert _code(_evict, e, **bad) == code, bad
    assert e.free_blocks() == free
    for s in (7, 8):
        assert e.seq_info(s) == (0, [])
    e.close()
    e = _engine(pool=None)
    e.seq_create(7)
    assert _code(_evict, e) == "STATE"
    e.close()


def test_evict_bytes():
    e = _engine()
    # [n][4] numbers, 7 + 3 source blocks, 2 + 1 destination blocks; 3 blocks of kept slots
    assert e.kv_evict_bytes([0, 1], [20, 3]) == 256 + 256
    for src, keep in (([5], [1]), ([0], [0]), ([0], [101])):
        assert e.kv_evict_bytes(src, keep) == 0
    e.close()
    with pytest.raises(vsk.VskError):
        _engine().kv_evict([7], [0, 1], [3], 0, 0, FAKE, 100, FAKE, 256, kept_ptr=FAKE)


def test_positions_and_prefixes_without_eviction_are_unchanged():
    e = _engine()
    e.batch_build([0, 2], [3, 17])
    b = e.batch_host()
    np.testing.assert_array_equal(b["pos"], list(range(97, 100)) + list(range(17)))
    e.seq_create(9)
    e.seq_share_prefix(9, 0, 96)
    assert e.seq_info(9)[0] == 96
    e.close()


def test_evict_refuses_metadata_among_its_buffers():
    e = _engine()
    e.seq_create(7)
    free = e.free_blocks()
    for bad in (dict(meta=FAKE), dict(mass=8 * FAKE + 256), dict(kept=8 * FAKE + 508), dict(mass_out=8 * FAKE),
                dict(slots=8 * FAKE + 128)):
        assert _code(_evict, e, **bad) == "ARG", bad
    assert e.free_blocks() == free and e.seq_info(7) == (0, [])
    e.close()
