"""The packed layer where its pool is short, on host tensors: the calls that would
launch something are left out, packing moves the blocks alone."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402
from tests.test_streaming_cpu import Streams  # noqa: E402

HQ, HKV, D, BS = 4, 2, 64, 16
BLOCK = 2 * HKV * BS * D * 2
LAYOUTS = [(HKV, D), (HKV, D | K.KV_Q4)]


class Backing:
    """Physical memory that is always there."""

    def map(self, off, n):
        return 0

    def unmap(self, off, n):
        return 0


class ElasticPool:
    """Virtual pages beyond what a limit or a shared budget lets be mapped, one bf16
    block (or three packed ones) a chunk."""

    def __init__(self, virtual, limit=0, budget=None, base=1 << 40):
        self.device = torch.device("cpu")
        self.handle = K.kv_pool_create_vmm(virtual * BLOCK, BS, LAYOUTS, (1 << 40) + (1 << 30), page_bytes=BLOCK // 32,
                                           chunk_bytes=BLOCK, physical_limit=limit * BLOCK, budget=budget, backend=Backing(),
                                           device_base=base)


class FixedPool:
    def __init__(self, n):
        self.device = torch.device("cpu")
        self.handle = K.kv_pool_create(1 << 40, n * BLOCK, BS, LAYOUTS, (1 << 40) + (1 << 30), page_bytes=BLOCK // 32)


def moved(t, packed, slots, keep, stream=None):
    """kv_seq_pack without its kernel: all or nothing."""
    bs = BS
    lens, done = t.lens(), packed.lens()
    to = {int(s): max(int(done[s]) // bs, max(0, int(lens[s]) - keep) // bs) for s in slots}
    n = sum(b - int(done[s]) // bs for s, b in to.items())
    K.kv_free_blocks(t.pool, 1, K.kv_alloc_blocks(t.pool, 1, n))
    for s, b in to.items():
        if b * bs > done[s]:
            packed.reserve(s, b * bs)
            packed.set_len(s, b * bs)
            t.evict(s, int(lens[s]) - b * bs, 0)
    return n


@pytest.fixture
def make(monkeypatch):
    from paper_2606_12950_gb300.streaming import PackedLayer

    Streams(monkeypatch)
    for name in ("kv_append_rotary", "paged_prompt_attn", "paged_decode_attn_q4", "kv_unpack_blocks"):
        monkeypatch.setattr(K, name, lambda *a, **kw: None)
    for name in ("kv_workspace_bytes", "kv_q4_workspace_bytes", "kv_prompt_workspace_bytes"):
        monkeypatch.setattr(K, name, lambda *a: 256)
    monkeypatch.setattr(K.SeqTab, "sync", lambda *a: None)
    monkeypatch.setattr(K.SeqTab, "pack", moved)
    made = []

    def layer(pool, S=2, max_tokens=400, keep=1):
        x = PackedLayer(0, HQ, HKV, D, BS, S, max_tokens, keep, K.kv_rotary_freqs(D), pool=pool)
        x.tab.pool = x.tab4.pool = pool.handle
        made.append((x, pool))
        return x

    yield layer
    for x, pool in made:
        x.tab4.close()
        x.tab.close()
        K.kv_pool_destroy(pool.handle)


def rows(n):
    return tuple(torch.zeros((n, h * D), dtype=torch.bfloat16) for h in (HQ, HKV, HKV))


def state(x):
    (a, b), (c, d) = x.tab.host(), x.tab4.host()
    st = K.kv_pool_stats(x.pool.handle)
    return a.tolist(), b.tolist(), c.tolist(), d.tolist(), st["blocks_used"]


@pytest.mark.parametrize("shared", [False, True])
def test_pages_stay_in_bf16_where_no_more_can_be_mapped(make, shared):
    """A limit, or another pool's share of a budget, refuses what the virtual range
    still has room for: prompts and steps go on, and a later call packs."""
    budget = K.kv_budget_create(9 * BLOCK) if shared else None
    x = make(ElasticPool(40, 0 if shared else 9, budget))
    if shared:
        other = ElasticPool(40, 0, budget, base=1 << 41)
        held = K.kv_alloc_blocks(other.handle, 0, 1)
        x.prompt([128, 0], *rows(128))            # eight pages, and the ninth is the other's
    else:
        x.prompt([128, 16], *rows(144))           # nine pages
    assert x.tab4.lens().tolist() == [0, 0] and x.tab.lens()[0] == 128
    if shared:
        K.kv_free_blocks(other.handle, 0, held)
        K.kv_pool_trim(other.handle)
    else:
        x.release(1)
    assert x.step(*rows(2)).shape == (2, HQ, D)   # takes the ninth page itself
    assert x.tab.lens()[0] == 129
    for n in range(130, 145):
        x.step(*rows(2))
        assert x.tab.lens()[0] == n
    assert x.tab4.lens()[0] == 0                  # all nine are full and in bf16
    x.release(0)
    x.prompt([97, 0], *rows(97))                  # seven pages: two for packing
    assert x.tab4.lens()[0] == 96 and x.packed_used() == 6 and x.pages_used() == 1
    if shared:
        K.kv_pool_destroy(other.handle)


def test_a_few_pages_at_a_time_under_a_limit(make):
    """Room for one superpage of packed pages: three, then those that they freed."""
    x = make(ElasticPool(100, 22))
    x.prompt([21 * BS, 0], *rows(21 * BS))
    assert x.tab4.lens()[0] == 20 * BS and x.pages_used() == 1 and x.packed_used() == 20


def test_a_refused_prompt_reserves_nothing(make):
    """The copies of packed pages are asked for before the new tokens' own pages: a
    prompt refused for want of them leaves tables and pool as they were."""
    x = make(FixedPool(8))
    x.prompt([100, 0], *rows(100))
    assert x.packed_used() == 6 and x.pages_used() == 1     # three superpages of eight
    hog = K.kv_alloc_blocks(x.pool.handle, 0, 3)
    before = state(x)
    with pytest.raises(K.KVError) as e:
        x.prompt([20, 0], *rows(20))                        # a page, and six for copies, of two
    assert e.value.code == K.KV_ERR_OUT_OF_BLOCKS
    assert state(x) == before
    K.kv_free_blocks(x.pool.handle, 0, hog)
    before = state(x)
    with pytest.raises(K.KVError):
        x.prompt([20, 30], *rows(50))
    assert state(x) == before
    x.release(0)
    x.prompt([60, 0], *rows(60))
    x.prompt([20, 0], *rows(20))                            # three copies, given back
    assert x.tab.lens()[0] == 80 and x.packed_used() == 4 and x.pages_used() == 1


def test_a_prompt_without_pages_of_its_own_gives_its_copies_back(make):
    x = make(FixedPool(8))
    x.prompt([100, 0], *rows(100))
    used = K.kv_pool_stats(x.pool.handle)["blocks_used"]
    with pytest.raises(K.KVError) as e:
        x.prompt([0, 400], *rows(400))                      # 25 pages
    assert e.value.code == K.KV_ERR_OUT_OF_BLOCKS
    assert K.kv_pool_stats(x.pool.handle)["blocks_used"] == used and x.tab.lens().tolist() == [100, 0]
    x.release(0)
    x.prompt([33, 0], *rows(33))
    used = K.kv_pool_stats(x.pool.handle)["blocks_used"]
    with pytest.raises(K.KVError):
        x.prompt([200, 0], *rows(200))                      # two copies, then 13 pages more
    assert K.kv_pool_stats(x.pool.handle)["blocks_used"] == used and x.tab.lens().tolist() == [33, 0]
