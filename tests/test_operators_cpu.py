"""Host parts of the rotary, window and page operators: frequencies and steps,
eviction from sequence tables, refusals before anything is launched."""
import math

import numpy as np
import pytest

from paper_2606_12950_gb300 import kvpool as K

FAKE_BASE = 1 << 40
FAKE_ERR = (1 << 40) + (1 << 30)


def pool(n_pages=64, layouts=((2, 64),), bs=16):
    block = min(2 * h * bs * d * 2 for h, d in layouts)
    return K.kv_pool_create(FAKE_BASE, n_pages * block, bs, list(layouts), FAKE_ERR)


def test_frequencies():
    f = K.kv_rotary_freqs(8, base=10000.0)
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001], rtol=1e-15)
    assert np.allclose(K.kv_rotary_freqs(8, scaling=K.KV_ROTARY_LINEAR, factor=4.0), f / 4, rtol=1e-15)
    g = K.kv_rotary_freqs(128, base=500000.0, scaling=K.KV_ROTARY_BY_PARTS, factor=8.0, original_len=8192,
                          low_turns=1.0, high_turns=4.0)
    f = K.kv_rotary_freqs(128, base=500000.0)
    turns = 8192 * f / (2 * math.pi)
    assert np.array_equal(g[turns >= 4], f[turns >= 4]) and np.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 4)
    keep = (turns[mid] - 1) / 3
    assert mid.any() and np.allclose(g[mid], keep * f[mid] + (1 - keep) * f[mid] / 8, rtol=1e-14)
    for kw in ({"rot_dim": 7}, {"rot_dim": 0}, {"rot_dim": 514}, {"base": 1.0}, {"base": math.nan},
               {"scaling": 1, "factor": 0.5}, {"scaling": 3}, {"scaling": 2, "factor": 2.0, "original_len": 0},
               {"scaling": 2, "factor": 2.0, "original_len": 8, "low_turns": 4.0, "high_turns": 4.0}):
        with pytest.raises(K.KVError):
            K.kv_rotary_freqs(**{"rot_dim": 8, **kw})


def test_steps_are_fractions_of_a_turn():
    f = np.array([2 * math.pi * x for x in (0.25, 0.5, 1.0, 1.75, -0.25, 0.0)])
    s = K.kv_rotary_steps(f)
    want = [0.25, 0.5, 0.0, 0.75, 0.75, 0.0]
    for a, w in zip(s, want):
        d = (float(a) / 2.0 ** 64 - w) % 1.0
        assert min(d, 1 - d) < 1e-15
    with pytest.raises(K.KVError):
        K.kv_rotary_steps([math.inf])
    with pytest.raises(K.KVError):
        K.kv_rotary_steps([])


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (17, 4), (32, 16), (33, 17), (100, 0), (10 ** 9, 3)])
def test_evict_gives_up_what_no_later_query_sees(window, sinks):
    h = pool()
    t = K.SeqTab(h, 0, 2, 12)
    t.reserve(0, 180)
    freed = 0
    for n in (0, 1, 40, 41, 100, 160, 161, 178):
        t.set_len(0, n)
        freed += t.evict(0, window, sinks)
        tab = t.host()[0][0]
        for b in range(12):
            # a token of the block is seen by the query at n - 1 or a later one
            seen = any(j < sinks or j > n - 1 - window for j in range(b * 16, b * 16 + 16))
            assert (tab[b] >= 0) == seen, (n, b)
        assert K.kv_pool_stats(h)["blocks_used"][0] == 12 - freed == t.counters()["blocks_held"]
    assert t.evict(0, window, sinks) == 0
    t.advance([0])  # the reach stays
    if freed:
        with pytest.raises(K.KVError):
            t.share_prefix(1, 0, 12)
    t.set_len(0, 20)
    t.trim(0)  # over given-up entries
    t.release(0)
    assert K.kv_pool_stats(h)["blocks_used"][0] == 0 and t.counters()["blocks_held"] == 0
    t.reserve(0, 192)
    t.close()
    K.kv_pool_destroy(h)


def test_evict_drops_one_reference():
    h = pool()
    t = K.SeqTab(h, 0, 3, 8)
    t.reserve(0, 128)
    t.set_len(0, 128)
    t.share_prefix(1, 0, 8)
    t.set_len(1, 128)
    assert t.evict(1, 16, 16) == 6
    assert K.kv_pool_stats(h)["blocks_used"][0] == 8
    assert t.evict(0, 16, 16) == 6
    assert K.kv_pool_stats(h)["blocks_used"][0] == 2
    st = t.replace([1], [32], [20])
    assert st[0] == 0 and K.kv_pool_stats(h)["blocks_used"][0] == 4
    t.close()
    K.kv_pool_destroy(h)


def test_refusals_on_the_host():
    h = pool()
    t = K.SeqTab(h, 0, 3, 8)
    for args in ((0, 0, 0), (0, 16, -1), (3, 16, 0), (-1, 16, 0)):
        with pytest.raises(K.KVError) as e:
            t.evict(*args)
        assert e.value.code == K.KV_ERR_INVALID_ARG
    t.reserve(0, 30)
    t.set_len(0, 16)
    t.fork(0, [1, 2])  # whole blocks: by reference alone
    assert (t.host()[0][1:, 0] == t.host()[0][0, 0]).all() and K.kv_block_refcount(h, int(t.host()[0][0, 0])) == 3
    for dsts in ([1], [0], [3]):
        with pytest.raises(K.KVError):
            t.fork(0, dsts)
    t.fork(0, [])
    with pytest.raises(K.KVError):
        K.kv_pool_compact(h, max_moves=-1)
    assert K.kv_pool_compact(h) == 0  # every superpage is one block
    with pytest.raises(K.KVError):
        K.kv_copy_blocks(h, 1, [0], [1])
    K.kv_pool_destroy(h)
    for call in (lambda: t.fork(0, [1]), lambda: t.evict(0, 4, 0)):
        with pytest.raises(K.KVError):
            call()  # the table's pool is gone
    t.close()


def test_numbers_of_numpy_and_wrong_ones():
    """Arguments as Python's or numpy's numbers; anything else is an error."""
    h = pool()
    R = K.Rotary(0, None)
    for n in (0, np.int64(0), np.int32(0)):
        K.kv_append_rotary(h, np.int64(0), R, None, np.int64(0), None, None, 0, None, 0, None, None, n, None, None,
                           np.int32(4), n, np.int64(0))
    with pytest.raises(K.KVError) as e:
        K.kv_append_rotary(h, 0, R, None, 0, None, None, 0, None, 0, None, None, np.int64(1), None, None, 4, 1, 0)
    assert e.value.code == K.KV_ERR_INVALID_ARG
    with pytest.raises(Exception):
        K.kv_append_rotary(h, 0, R, None, "x", None, None, 0, None, 0, None, None, 0, None, None, 4, 0, 0)
    K.kv_pool_destroy(h)
