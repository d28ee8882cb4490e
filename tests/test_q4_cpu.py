"""Host parts of the 4-bit blocks and the normed append: geometry, tables,
refusals before anything is launched."""
import numpy as np
import pytest

from paper_2606_12950_gb300 import kvpool as K

BASE, ERR, X = 1 << 40, (1 << 40) + (1 << 30), 1 << 41


def pool(supers=12, Hkv=2, d=64, bs=16, layouts=None, page=None, **kw):
    block = 2 * Hkv * bs * d * 2
    return K.kv_pool_create(BASE, supers * block, bs, layouts or [(Hkv, d), (Hkv, d | K.KV_Q4)], ERR,
                            page_bytes=block // 32 if page is None else page, **kw)


def code(call, *args):
    with pytest.raises(K.KVError) as e:
        call(*args)
    return e.value.code


def test_a_superpage_holds_one_bf16_block_or_three_packed_ones():
    h = pool()
    assert K.kv_pool_stats(h)["blocks_capacity"][:2] == [12, 36]
    a, b = K.kv_alloc_blocks(h, 0, 4), K.kv_alloc_blocks(h, 1, 24)
    assert set(a % 32) == {0} and set(b % 32) == {0, 9, 18}
    spans = sorted([(int(i), int(i) + 32) for i in a] + [(int(i), int(i) + 9) for i in b])
    assert all(x[1] <= y[0] for x, y in zip(spans, spans[1:])) and spans[-1][1] <= 12 * 32
    st = K.kv_pool_stats(h)
    assert st["bytes_used"] == (4 * 32 + 24 * 9) * 256
    assert code(K.kv_alloc_blocks, h, 0, 1) == K.KV_ERR_OUT_OF_BLOCKS
    K.kv_free_blocks(h, 1, b[:3])
    K.kv_pool_trim(h)
    assert len(K.kv_alloc_blocks(h, 0, 1)) == 1  # the superpage serves the other kind
    K.kv_pool_destroy(h)


def test_pools_of_packed_blocks_alone():
    K.kv_pool_destroy(pool(Hkv=1))  # pages of 128 bytes
    h = pool(layouts=[(2, 64 | K.KV_Q4)], page=0)
    assert K.kv_pool_stats(h)["pages_total"] == 12 * 32 // 9
    K.kv_pool_destroy(h)


def test_geometry_refusals():
    for kw in ({"layouts": [(2, 64), (2, 80 | K.KV_Q4)]}, {"bs": 24}, {"page": 64}, {"page": 512}):
        assert code(lambda kw=kw: pool(**kw)) == K.KV_ERR_INVALID_ARG
    # without a 4-bit layout, superpages are whole blocks as ever
    assert code(lambda: pool(layouts=[(2, 64), (3, 64)], page=4096)) == K.KV_ERR_INVALID_ARG


def test_the_bf16_calls_refuse_packed_layouts():
    h, Q = pool(), 1
    U = K.KV_ERR_UNSUPPORTED
    assert code(K.kv_append, h, Q, X, X, X, X, 4, 1) == U
    assert code(K.kv_append_rotary, h, Q, K.Rotary(0, None), X, 512, X, None, 0, None, 0, None, None, 1, X, X, 4, 1, 4) == U
    assert code(K.kv_append_rotary_norm, h, Q, K.Rotary(0, None), K.HeadNorm(X, X), X, 512, X, None, 0, None, 0, None, None,
                1, X, X, 4, 1, 4) == U
    assert code(K.kv_workspace_bytes, h, Q, 1, 4, 4) == U
    assert code(K.paged_decode_attn, h, Q, X, X, X, X, 4, 1, 4, 0.1, 0, X, 1 << 30) == U
    assert code(K.paged_decode_attn_window, h, Q, X, None, None, X, X, X, 4, 1, 4, 0.1, 8, 0, 0, X, 1 << 30) == U
    assert code(K.kv_prompt_workspace_bytes, h, Q, 1, 4, 1, 1, 4, 0, 0) == U
    assert code(K.kv_cascade_workspace_bytes, h, Q, 1, 4, 4) == U
    b = K.kv_alloc_blocks(h, 1, 2)
    assert code(K.kv_copy_blocks, h, 1, b[:1], b[1:], [5]) == U
    t = K.SeqTab(h, 1, 2, 4)
    t.reserve(0, 32)
    t.set_len(0, 20)
    assert code(t.fork, 0, [1]) == U
    t.set_len(0, 32)
    t.fork(0, [1])  # by reference
    t.close()
    K.kv_pool_destroy(h)


def test_pack_refusals():
    h = pool(layouts=[(2, 64), (2, 64 | K.KV_Q4), (1, 64 | K.KV_Q4), (4, 64)], bs=32, page=256)
    a, b = K.kv_alloc_blocks(h, 0, 3), K.kv_alloc_blocks(h, 1, 3)
    I, U = K.KV_ERR_INVALID_ARG, K.KV_ERR_UNSUPPORTED
    for call, x, y, lx, ly in ((K.kv_pack_blocks, a, b, 0, 1), (K.kv_unpack_blocks, b, a, 1, 0)):
        assert code(call, h, lx, lx, x, x) == U and code(call, h, ly, lx, x, y) == U
        assert code(call, h, 9, ly, x, y) == I and code(call, h, lx, -1, x, y) == I
        assert code(call, h, lx, ly, x[:2], [y[0], y[0]]) == I        # a destination twice
        assert code(call, h, lx, ly, [x[0], 5], y[:2]) == I           # not a live block
        assert code(call, h, lx, ly, y[:2], y[1:]) == I               # of the other kind
        assert code(call, h, lx, ly, [-1], y[:1]) == I and code(call, h, lx, ly, [1 << 30], y[:1]) == I
        call(h, lx, ly, [], [])
        with pytest.raises(ValueError):
            call(h, lx, ly, x, y[:2])
    assert code(K.kv_pack_blocks, h, 0, 2, a, b) == I and code(K.kv_pack_blocks, h, 3, 1, a, b) == I  # other heads
    assert code(K.kv_pack_blocks, None, 0, 1, a, b) == I
    K.kv_free_blocks(h, 1, b[2:])
    assert code(K.kv_pack_blocks, h, 0, 1, a, b) == I
    K.kv_pool_destroy(h)


def state(t):
    table, lens = t.host()
    return table.tolist(), lens.tolist(), t.counters()["blocks_held"]


def test_seq_pack_refusals_leave_both_tables():
    h = pool()
    t, q = K.SeqTab(h, 0, 3, 6), K.SeqTab(h, 1, 3, 3)
    t.reserve(0, 60)
    t.set_len(0, 60)
    t.reserve(1, 90)
    t.set_len(1, 90)
    I = K.KV_ERR_INVALID_ARG
    before = state(t), state(q), K.kv_pool_stats(h)
    assert code(t.pack, q, [0], 0) == I and code(t.pack, q, [0, 0], 1) == I
    assert code(t.pack, q, [3], 1) == I and code(t.pack, q, [-1], 1) == I
    assert code(t.pack, q, [1], 1) == I            # five blocks: the other table holds three
    assert code(q.pack, t, [0], 1) == K.KV_ERR_UNSUPPORTED
    other = K.SeqTab(h, 1, 2, 6)
    assert code(t.pack, other, [0], 1) == I        # other slots
    assert t.pack(q, [], 1) == 0 and t.pack(q, [0, 2], 60) == 0 and t.pack(q, [0], 45) == 0  # nothing full enough
    assert (state(t), state(q), K.kv_pool_stats(h)) == before
    q.reserve(0, 16)                               # held, but no packed tokens
    assert code(t.pack, q, [0], 1) == I
    q.set_len(0, 10)                               # no whole blocks
    assert code(t.pack, q, [0], 1) == I
    q.release(0)
    t.evict(0, 16, 0)                              # blocks given up
    assert code(t.pack, q, [0], 1) == I
    hog = K.kv_alloc_blocks(h, 0, K.kv_pool_stats(h)["blocks_capacity"][0] - K.kv_pool_stats(h)["blocks_used"][0])
    K.kv_alloc_blocks(h, 1, K.kv_pool_stats(h)["blocks_cached"][1])
    before = state(t), state(q), K.kv_pool_stats(h)
    assert code(t.pack, q, [1], 42) == K.KV_ERR_OUT_OF_BLOCKS
    assert (state(t), state(q), K.kv_pool_stats(h)) == before
    K.kv_free_blocks(h, 0, hog)
    K.kv_pool_destroy(h)
    assert code(t.pack, q, [1], 42) == I           # the pool is gone
    for x in (t, q, other):
        x.close()


def test_seq_pack_without_a_gpu_changes_nothing():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("the launch would run over an address that is no memory")
    h = pool()
    t, q = K.SeqTab(h, 0, 2, 6), K.SeqTab(h, 1, 2, 6)
    t.reserve(0, 60)
    t.set_len(0, 60)
    before = state(t), state(q), K.kv_pool_stats(h)["blocks_used"]
    assert code(t.pack, q, [0], 1) == K.KV_ERR_CUDA
    assert (state(t), state(q), K.kv_pool_stats(h)["blocks_used"]) == before
    for x in (t, q):
        x.close()
    K.kv_pool_destroy(h)


def test_norm_refusals():
    h = pool(layouts=[(2, 64), (1, 512)], page=8192)
    R, I = K.Rotary(0, None), K.KV_ERR_INVALID_ARG

    def call(norm, layout=0, T=1, q=X):
        K.kv_append_rotary_norm(h, layout, R, norm, q, 4 * (64, 512)[layout], X, None, 0, None, 0, None, None, T, X, X, 4, T, 4)

    for bad in (K.HeadNorm(X, X, eps=-1.0), K.HeadNorm(X, X, eps=float("nan")), K.HeadNorm(X, X, eps=float("inf")),
                K.HeadNorm(X + 2, X), K.HeadNorm(X, X + 8), K.HeadNorm(X, X, offset=float("nan"))):
        assert code(call, bad) == I
    assert code(call, K.HeadNorm(X, X), 1) == K.KV_ERR_UNSUPPORTED
    assert code(call, K.HeadNorm(X, X), 0, 1, None) == I
    call(K.HeadNorm(X, X), T=0)
    assert K.lib().kv_append_rotary_norm(h, 0, R.address, None, X, 256, X, None, 0, None, 0, None, None, 0, X, X, 4, 0, 4,
                                         None) == I
    K.kv_pool_destroy(h)


def test_attention_refusals():
    h = pool()
    I, U = K.KV_ERR_INVALID_ARG, K.KV_ERR_UNSUPPORTED

    def call(layout=0, q4=1, q=X, k=None, v=None, out=X, mb=4, mb4=4, S=1, Hq=4, scale=0.1, table=X, table4=X):
        K.paged_decode_attn_q4(h, layout, q4, q, k, v, out, table, X, mb, table4, X, mb4, S, Hq, scale, X, 1 << 30)

    assert code(lambda: call(layout=1)) == U and code(lambda: call(q4=0)) in (U, K.KV_ERR_CUDA)
    for kw in ({"layout": 7}, {"q4": -1}, {"Hq": 3}, {"mb": 0}, {"mb4": 0}, {"S": -1}, {"scale": float("nan")},
               {"mb": 1 << 28}, {"mb4": 1 << 28}):
        assert code(lambda kw=kw: call(**kw)) == I
    assert code(lambda: call(Hq=6)) == U  # three heads a KV head
    assert code(K.kv_q4_workspace_bytes, h, 0, 1, 4, 4) == U and code(K.kv_q4_workspace_bytes, h, 1, 1, 3, 4) == I
    K.kv_pool_destroy(h)


def test_vmm_pools_and_layouts_of_several_models():
    """Chunks follow superpages of three packed blocks; two models' packed and bf16
    blocks in one pool."""
    class Backing:
        def __init__(self):
            self.mapped = set()

        def map(self, off, n):
            self.mapped.add(off)
            return 0

        def unmap(self, off, n):
            self.mapped.remove(off)
            return 0

    fb, block = Backing(), 2 * 2 * 16 * 64 * 2
    layouts = [(2, 64), (2, 64 | K.KV_Q4), (4, 64), (4, 64 | K.KV_Q4)]
    h = K.kv_pool_create_vmm(16 * block, 16, layouts, ERR, page_bytes=block // 32, chunk_bytes=2 * block, backend=fb,
                             device_base=BASE)
    # a superpage holds the largest block, 64 pages: one, two, three (18) or seven (9) blocks
    assert K.kv_pool_stats(h)["blocks_capacity"] == [16, 8 * 7, 8, 8 * 3]
    a = K.kv_alloc_blocks(h, 1, 8)
    assert len(fb.mapped) == 2 and len(set(a)) == 8 and set(a % 64) <= set(range(0, 63, 9))
    b = K.kv_alloc_blocks(h, 3, 4)
    assert set(b % 64) <= {0, 18, 36} and len(fb.mapped) == 4
    spans = sorted([(int(i), int(i) + 9) for i in a] + [(int(i), int(i) + 18) for i in b])
    assert all(x[1] <= y[0] for x, y in zip(spans, spans[1:]))
    K.kv_free_blocks(h, 1, a)
    K.kv_free_blocks(h, 3, b[:3])
    K.kv_pool_trim(h)
    assert len(fb.mapped) == 1
    c = K.kv_alloc_blocks(h, 2, 7)
    assert len(fb.mapped) == 8 and code(K.kv_alloc_blocks, h, 0, 1) == K.KV_ERR_OUT_OF_BLOCKS
    K.kv_free_blocks(h, 2, c)
    K.kv_free_blocks(h, 3, b[3:])
    K.kv_pool_trim(h)
    assert not fb.mapped
    K.kv_pool_destroy(h)
