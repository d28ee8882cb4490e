"""Page copies, forks and compaction on the device: contents, tables and
allocator afterwards."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402
from paper_2606_12950_gb300.runner import DevicePool, VmmPool  # noqa: E402

pytestmark = pytest.mark.gpu


def pool_of(n_pages, Hkv=2, d=64, bs=16, seed=0, layouts=None):
    layouts = layouts or [(Hkv, d)]
    page = min(2 * h * bs * x * 2 for h, x in layouts)
    p = DevicePool(n_pages, page, bs, layouts, shuffle_seed=seed)
    bits = torch.randint(-2 ** 15, 2 ** 15, (p.buf.numel() // 2,), dtype=torch.int16, device="cuda")
    p.buf.view(torch.int16).copy_(bits)
    return p


def pages(p, Hkv=2, d=64, bs=16):
    return p.buf.view(torch.int16).view(-1, 2, Hkv, bs, d)


@pytest.mark.parametrize("n", [1, 5, 81, 400, 3000])
@pytest.mark.parametrize("Hkv,d,bs", [(2, 64, 16), (8, 128, 16), (1, 8, 16), (3, 24, 7)])
@pytest.mark.parametrize("partial", [False, True])
def test_copies_any_bits(n, Hkv, d, bs, partial):
    page = 2 * Hkv * bs * d * 2
    if page % 256:
        pytest.skip("no whole page")
    p = pool_of(2 * n + 5, Hkv, d, bs)
    ids = K.kv_alloc_blocks(p.handle, 0, 2 * n + 5)
    rng = np.random.default_rng(n)
    ids = rng.permutation(ids)
    src, dst = ids[:n].copy(), ids[n : 2 * n].copy()
    src[-1] = src[0]  # a source may appear twice
    tokens = rng.integers(0, bs + 1, n) if partial else None
    want = pages(p, Hkv, d, bs).clone()
    for i in range(n):
        m = int(tokens[i]) if partial else bs
        want[dst[i], :, :, :m] = want[src[i], :, :, :m]
    K.kv_copy_blocks(p.handle, 0, src, dst, tokens)
    src[:] = 0  # the arrays are the caller's again
    assert torch.equal(pages(p, Hkv, d, bs), want)
    p.close()


def test_copy_refusals():
    p = pool_of(12)
    a = K.kv_alloc_blocks(p.handle, 0, 6)
    free = [i for i in range(12) if i not in a][0]
    before = p.buf.clone()
    for src, dst, tok in ([a[0]], [free], None), ([free], [a[0]], None), ([a[0], a[1]], [a[2], a[2]], None), \
            ([a[0], a[1]], [a[1], a[2]], None), ([a[0]], [a[1]], [17]), ([a[0]], [a[1]], [-1]), ([-1], [a[1]], None), \
            ([a[0]], [12], None), ([a[0]], [a[0]], None):
        with pytest.raises(K.KVError) as e:
            K.kv_copy_blocks(p.handle, 0, src, dst, tok)
        assert e.value.code == K.KV_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        K.kv_copy_blocks(p.handle, 0, a[:2], a[2:3])
    K.kv_copy_blocks(p.handle, 0, [], [])
    torch.cuda.synchronize()
    assert torch.equal(before, p.buf)
    K.kv_free_blocks(p.handle, 0, a)  # the refused calls left the pool's marks clean
    p.close()


@pytest.mark.parametrize("length", [1, 15, 16, 17, 40, 64])
def test_fork_and_diverge(length):
    p = pool_of(64)
    t = K.SeqTab(p.handle, 0, 6, 8)
    t.reserve(0, 100)
    t.set_len(0, length)
    t.fork(0, [2, 4, 5])
    tab, lens = t.host()
    full, tail = divmod(length, 16)
    for d in (2, 4, 5):
        assert lens[d] == length
        assert (tab[d, :full] == tab[0, :full]).all()
        if tail:
            assert tab[d, full] not in tab[0] and K.kv_block_refcount(p.handle, int(tab[d, full])) == 1
            got, want = pages(p)[int(tab[d, full])], pages(p)[int(tab[0, full])]
            assert torch.equal(got[:, :, :tail], want[:, :, :tail])
        assert (tab[d, full + (tail > 0):] == -1).all()
    if full:
        assert K.kv_block_refcount(p.handle, int(tab[0, 0])) == 4
    held = t.counters()["blocks_held"]
    assert held == 7 + 3 * (full + (tail > 0))
    # every slot goes on by itself
    t.advance([0, 2, 4])
    for s in (0, 2, 4, 5):
        t.release(s)
    assert K.kv_pool_stats(p.handle)["blocks_used"][0] == 0
    t.close()
    p.close()


def test_fork_all_or_nothing():
    p = pool_of(5)
    t = K.SeqTab(p.handle, 0, 6, 4)
    t.reserve(0, 40)  # 3 blocks: 2 free
    t.set_len(0, 37)
    before = t.host()
    with pytest.raises(K.KVError) as e:
        t.fork(0, [1, 2, 3])
    assert e.value.code == K.KV_ERR_OUT_OF_BLOCKS
    for dsts in ([0], [1, 1], [9], [-1]):
        with pytest.raises(K.KVError) as e:
            t.fork(0, dsts)
        assert e.value.code == K.KV_ERR_INVALID_ARG
    after = t.host()
    assert all((x == y).all() for x, y in zip(before, after))
    assert K.kv_pool_stats(p.handle)["blocks_used"][0] == 3
    t.fork(0, [1, 2])
    with pytest.raises(K.KVError):
        t.fork(0, [1])  # not empty
    t.close()
    p.close()


def test_fork_of_an_evicted_chat():
    p = pool_of(64)
    t = K.SeqTab(p.handle, 0, 3, 16)
    t.reserve(0, 200)
    t.set_len(0, 200)
    assert t.evict(0, 50, 4) == 8  # blocks 1..8: 9 * 16 = 144 <= 150
    t.fork(0, [1])
    tab, _ = t.host()
    assert (tab[1, 1:9] == -1).all() and (tab[1, :1] == tab[0, :1]).all() and (tab[1, 9:12] == tab[0, 9:12]).all()
    t.release(0)
    t.release(1)
    assert K.kv_pool_stats(p.handle)["blocks_used"][0] == 0
    t.close()
    p.close()


def contents(p, tabs, view):
    """What each table's tokens read, by slot."""
    torch.cuda.synchronize()
    out = []
    for t in tabs:
        tab, lens = t.host()
        for s in range(t.S):
            ids = [int(x) for x in tab[s] if x >= 0]
            out.append(view(t, ids))
    return out


def test_compact_superpages_of_two_layouts():
    """Blocks of a small layout scattered over superpages move together, and
    whole superpages come back to the other layout."""
    layouts = [(8, 64), (2, 64)]  # 4 small blocks a superpage
    p = pool_of(4 * 40, bs=16, layouts=layouts, seed=3)
    small = K.SeqTab(p.handle, 1, 40, 8)
    other = K.SeqTab(p.handle, 1, 4, 8)
    rng = np.random.default_rng(1)
    for s in range(40):
        small.reserve(s, 16 * 4)
        small.set_len(s, 50)
    for s in rng.permutation(40)[:26]:
        small.release(int(s))
    for s in range(40):
        if small.lens()[s]:
            small.set_len(s, 33)
            small.trim(s)
    other.reserve(0, 16)
    other.share_prefix(1, 0, 1)  # a block of another table, referenced twice
    pinned = K.kv_alloc_blocks(p.handle, 1, 1)  # no table's: it stays
    view = lambda t, ids: p.buf.view(4 * 40, -1)[ids].clone()  # noqa: E731
    pin_before = view(None, [int(pinned[0])])
    before, st0 = contents(p, [small, other], view), K.kv_pool_stats(p.handle)
    refs = {int(b) for b in other.host()[0].ravel() if b >= 0}
    K.kv_pool_trim(p.handle)
    un0 = K.kv_pool_stats(p.handle)["pages_unassigned"]
    assert K.kv_pool_compact(p.handle, max_moves=0) == 0
    moved = K.kv_pool_compact(p.handle)
    assert moved > 0
    K.kv_pool_trim(p.handle)
    st1 = K.kv_pool_stats(p.handle)
    after = contents(p, [small, other], view)
    assert all(torch.equal(a, b) for a, b in zip(before, after))
    assert torch.equal(pin_before, view(None, [int(pinned[0])]))
    assert st1["blocks_used"] == st0["blocks_used"] and st1["pages_unassigned"] > un0
    # as packed as whole superpages allow, the pinned block's aside
    used = st1["blocks_used"][1]
    assert 160 - st1["pages_unassigned"] <= 4 * (-(-used // 4) + 1)
    tab = np.concatenate([small.host()[0].ravel(), other.host()[0].ravel()])
    live = [int(b) for b in tab if b >= 0]
    assert len(set(live)) == used - 1 and int(pinned[0]) not in live
    for b in set(live):
        assert K.kv_block_refcount(p.handle, b) == live.count(b)
    assert len(refs) == 1
    # moved entries reach the device with the next sync
    dev, lens = torch.full((40, 8), -7, dtype=torch.int32, device="cuda"), torch.zeros(40, dtype=torch.int32, device="cuda")
    small.sync(dev, lens)
    assert (dev.cpu().numpy() == small.host()[0]).all()
    assert K.kv_pool_compact(p.handle) == 0  # nothing left to gain
    for s in range(40):
        small.release(s)
    small.close()
    other.close()
    K.kv_free_blocks(p.handle, 1, pinned)
    assert K.kv_pool_stats(p.handle)["blocks_used"] [1] == 0
    K.kv_pool_trim(p.handle)
    assert len(K.kv_alloc_blocks(p.handle, 0, 40)) == 40  # every superpage is whole again
    p.close()


@pytest.mark.parametrize("trim_first", [False, True])
def test_compact_gives_physical_memory_back(trim_first):
    """A VMM pool's chunks, also where freed superpages are in the shared list."""
    page = 2 * 2 * 16 * 64 * 2
    gran = 2 << 20
    p = VmmPool(16 * gran, page, 16, [(2, 64)], chunk_bytes=gran)
    per = gran // page
    t = K.SeqTab(p.handle, 0, 8 * 4, per // 4)
    rng = np.random.default_rng(0)
    for s in range(32):
        t.reserve(s, 16 * (per // 4))
        t.set_len(s, 16 * (per // 4))
    ids = [int(x) for x in t.host()[0].ravel()]
    p.fill_random(ids, 5)
    for s in rng.permutation(32)[:20]:
        t.release(int(s))
    if trim_first:
        p.trim()
    mapped = p.stats()["bytes_mapped"]
    tab0 = t.host()[0]
    before = [p.read_pages([int(x) for x in row if x >= 0]) for row in tab0 if (row >= 0).any()]
    moved = K.kv_pool_compact(p.handle)
    assert moved > 0
    p.trim()
    assert p.stats()["bytes_mapped"] == 3 * gran < mapped
    tab1 = t.host()[0]
    after = [p.read_pages([int(x) for x in row if x >= 0]) for row in tab1 if (row >= 0).any()]
    assert all((a == b).all() for a, b in zip(before, after))
    for s in range(32):
        if t.lens()[s]:
            t.release(s)
    p.trim()
    assert p.stats()["bytes_mapped"] == 0
    for s in range(32):
        t.reserve(s, 16 * (per // 4))  # everything can be had again
    t.close()
    p.close()
