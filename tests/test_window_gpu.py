"""Windowed decode attention against its definition in 64 bits: windows and
sinks at and around tile and block edges, evicted blocks, NaN wherever a token
is unseen, all head layouts, splits, fused appends."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


def attend(c, q, window, sinks, k=None, v=None, splits=0, scale=None, stream=None):
    out = torch.full((c.S, c.Hq, c.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    nb = max(256, K.kv_workspace_bytes(c.h, 0, c.S, c.Hq, c.max_blocks, splits))
    ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda")
    K.paged_decode_attn_window(c.h, 0, q, k, v, out, c.table, c.lens, c.max_blocks, c.S, c.Hq,
                               c.d ** -0.5 if scale is None else scale, window, sinks, splits, ws, nb, stream)
    torch.cuda.synchronize()
    return out


def case(n, Hq, Hkv, d, bs, window, sinks, seed=0, evict=True):
    from tests.paged_ref import Paged, holds

    nq = np.ones(len(n), np.int64)
    return Paged(n, nq, Hq, Hkv, d, bs, seed, held=holds(n, nq, window, sinks, bs) if evict else None)


def verify(c, q, window, sinks, **kw):
    from tests.paged_ref import check

    # an empty sequence's row is zero; the reference leaves it so
    ref, bound = c.reference(q, kw.get("scale") or c.d ** -0.5, window, sinks)
    out = attend(c, q, window, sinks, **kw)
    check(out, ref, bound)
    assert c.error() == 0
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (15, 4), (16, 0), (17, 16), (31, 33), (32, 5), (64, 64),
                                          (100, 0), (300, 7), (5000, 3)])
def test_windows_and_sinks(d, window, sinks):
    n = [1, 2, 15, 16, 17, 33, 64, 65, 100, 131, 500, 777]
    c = case(n, 8, 2, d, 16, window, sinks, seed=window + sinks)
    verify(c, c.normal(c.S, 8, d), window, sinks)
    c.close()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 2), (8, 2), (10, 2), (8, 1), (3, 3)])
@pytest.mark.parametrize("d,bs", [(64, 16), (64, 48), (128, 16), (128, 64), (128, 256)])
def test_head_layouts_and_blocks(Hq, Hkv, d, bs):
    n = [700, 3, 260, 1201]
    c = case(n, Hq, Hkv, d, bs, 200, 10, seed=Hq * 100 + bs)
    verify(c, c.normal(c.S, Hq, d), 200, 10)
    c.close()


@pytest.mark.parametrize("splits", [0, 1, 7, 500])
def test_one_long_sequence_and_splits(splits):
    c = case([20011], 8, 2, 128, 16, 4096, 4, seed=splits)
    verify(c, c.normal(1, 8, 128), 4096, 4, splits=splits)
    c.close()


@pytest.mark.parametrize("scale", [1.0, -0.3, 0.0])
def test_scales(scale):
    from tests.paged_ref import check

    c = case([90, 300], 8, 2, 128, 16, 64, 4)
    q = c.normal(2, 8, 128)
    ref, bound = c.reference(q, scale, 64, 4)
    check(attend(c, q, 64, 4, scale=scale), ref, bound)
    c.close()


def test_many_sequences_some_empty():
    rng = np.random.default_rng(5)
    n = rng.integers(0, 400, 700)
    n[::13] = 0
    c = case(n, 8, 2, 64, 16, 50, 20, seed=9)
    verify(c, c.normal(c.S, 8, 64), 50, 20)
    c.close()


@pytest.mark.parametrize("d,bs", [(64, 16), (64, 64), (128, 32)])
@pytest.mark.parametrize("window,sinks", [(16, 0), (33, 4), (1000, 2), (0, 0)])
def test_fused_append(d, bs, window, sinks):
    n = [1, 16, 17, 48, 49, 333, 512]
    c = case(n, 10, 2, d, bs, window, sinks, seed=bs)
    k, v, q = c.normal(c.S, 2, d), c.normal(c.S, 2, d), c.normal(c.S, 10, d)
    want = c.pool.clone()
    for s, m in enumerate(n):
        b = c.host_table[s, (m - 1) // bs]
        want[b, 0, :, (m - 1) % bs], want[b, 1, :, (m - 1) % bs] = k[s], v[s]
    out = attend(c, q, window, sinks, k=k, v=v)
    assert torch.equal(c.pool.view(torch.int16), want.view(torch.int16))
    from tests.paged_ref import check

    check(out, *c.reference(q, d ** -0.5, window, sinks))
    assert c.error() == 0
    c.close()


def test_whole_context_is_the_plain_call():
    c = case([700, 90, 16], 8, 2, 128, 16, 0, 0)
    q = c.normal(3, 8, 128)
    out = torch.empty_like(q)
    nb = K.kv_workspace_bytes(c.h, 0, 3, 8, c.max_blocks, 0)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    K.paged_decode_attn(c.h, 0, q, out, c.table, c.lens, c.max_blocks, 3, 8, 128 ** -0.5, 0, ws, nb)
    for window in (0, c.max_blocks * 16, 10 ** 9):
        assert torch.equal(attend(c, q, window, 5), out)
    c.close()


def test_infinities_and_nan_unseen_and_seen():
    """Unseen rows hold NaN (the pool's fill) and infinities; a seen NaN reaches
    its own sequence alone."""
    c = case([120, 120], 8, 2, 128, 16, 32, 4, seed=1, evict=False)
    b = c.host_table
    c.pool[b[0, 2], :, :, :] = float("inf")   # tokens 32..47: between the sinks and the window
    c.pool[b[0, 0], :, :, 4:] = float("-inf")  # the sinks' block past the sinks
    q = c.normal(2, 8, 128)
    verify(c, q, 32, 4)
    c.pool[b[1, 7], 1, 0, 3, 5] = float("nan")  # seen: token 115, V of KV head 0
    out = attend(c, q, 32, 4)
    bad = torch.isnan(out)
    assert bad[1, :4, 5].all() and bad.sum() == 4
    c.close()


def test_step_overlap_gives_the_same_bits():
    from tests.paged_ref import Paged, holds

    n = np.array([5000, 700, 90, 2000] * 8)
    c = Paged(n, np.ones(32, np.int64), 32, 8, 128, 16, 4, held=holds(n, np.ones(32), 1024, 4, 16))
    nb = K.kv_workspace_bytes(c.h, 0, 32, 32, c.max_blocks, 0)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    qs = [c.normal(32, 32, 128) for _ in range(6)]
    got = {}
    for on in (False, True):
        K.kv_set_attn_step_overlap(c.h, on)
        outs = [torch.empty_like(q) for q in qs]
        for q, o in zip(qs, outs):
            K.paged_decode_attn_window(c.h, 0, q, None, None, o, c.table, c.lens, c.max_blocks, 32, 32, 0.1, 1024, 4,
                                       0, ws, nb)
        torch.cuda.synchronize()
        got[on] = torch.stack(outs)
    assert torch.equal(got[False], got[True])
    assert K.kv_pool_stats(c.h)["attn_calls_overlapped"] >= 5
    c.close()


def test_cuda_core_variant_of_the_pool_leaves_the_call_alone():
    c = case([300, 5], 8, 2, 128, 16, 64, 4)
    K.kv_set_attn_variant(c.h, 1)
    verify(c, c.normal(2, 8, 128), 64, 4)
    c.close()


def test_refusals():
    c = case([100], 8, 2, 128, 16, 64, 4)
    q = c.normal(1, 8, 128)
    for kw in ({"window": -1}, {"sinks": -1}, {"scale": float("inf")}):
        with pytest.raises(K.KVError) as e:
            attend(c, q, kw.get("window", 64), kw.get("sinks", 4), scale=kw.get("scale"))
        assert e.value.code == K.KV_ERR_INVALID_ARG
    with pytest.raises(K.KVError) as e:
        K.paged_decode_attn_window(c.h, 0, q, None, None, q, c.table, c.lens, c.max_blocks, 1, 8, 1.0, 64, 4, 0, None, 0)
    assert e.value.code == K.KV_ERR_WORKSPACE
    with pytest.raises(K.KVError):
        attend(c, q, 64, 4, k=q)  # K without V
    c.table[0, 6] = 10 ** 6  # the window's block outside the pool: reported, not touched
    attend(c, q, 64, 4)
    assert c.error() == K.KV_ERR_DEVICE_BOUNDS
    c.close()
