"""Prompt chunks' attention against its definition in 64 bits: ragged chunks,
windows and sinks, NaN in every unseen place, NaN and infinities in seen ones."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


def attend(c, q, window, sinks, scale=None, max_q=None, stream=None):
    out = torch.full((c.T, c.Hq, c.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    max_q = int(c.nq.max()) if max_q is None else max_q
    nb = K.kv_prompt_workspace_bytes(c.h, 0, c.S, c.Hq, c.T, max_q, c.max_blocks, window, sinks)
    ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda") if nb else None
    K.paged_prompt_attn(c.h, 0, q, out, c.starts, c.T, max_q, c.table, c.lens, c.max_blocks, c.S, c.Hq,
                        c.d ** -0.5 if scale is None else scale, window, sinks, ws, nb, stream)
    torch.cuda.synchronize()
    return out


def case(n, nq, Hq, Hkv, d, bs, window, sinks, seed=0, evict=True, **kw):
    from tests.paged_ref import Paged, holds

    return Paged(n, nq, Hq, Hkv, d, bs, seed, held=holds(n, nq, window, sinks, bs) if evict else None, **kw)


def verify(c, q, window, sinks, scale=None, **kw):
    from tests.paged_ref import check

    ref, bound = c.reference(q, c.d ** -0.5 if scale is None else scale, window, sinks)
    out = attend(c, q, window, sinks, scale=scale, **kw)
    check(out, ref, bound)
    assert c.error() == 0
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 2), (16, 16), (100, 4), (128, 0), (129, 130), (300, 1)])
def test_windows_and_sinks(d, window, sinks):
    n, nq = [1, 40, 128, 129, 400, 700, 9], [1, 40, 100, 129, 7, 300, 0]
    c = case(n, nq, 8, 2, d, 16, window, sinks, seed=window + sinks)
    verify(c, c.normal(c.T, 8, d), window, sinks)
    c.close()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 2), (8, 2), (10, 2), (8, 1), (3, 3)])
@pytest.mark.parametrize("d,bs", [(64, 16), (64, 256), (128, 16), (128, 48), (128, 128)])
@pytest.mark.parametrize("window", [0, 150])
def test_head_layouts_and_blocks(Hq, Hkv, d, bs, window):
    n, nq = [330, 65, 200], [290, 65, 20]
    c = case(n, nq, Hq, Hkv, d, bs, window, 5, seed=Hq * 100 + bs)
    verify(c, c.normal(c.T, Hq, d), window, 5)
    c.close()


@pytest.mark.parametrize("window", [0, 2000])
def test_few_rows_on_a_long_context(window):
    """The key range is split and merged."""
    c = case([9001], [6], 8, 2, 128, 16, window, 4, seed=3)
    q = c.normal(6, 8, 128)
    assert K.kv_prompt_workspace_bytes(c.h, 0, 1, 8, 6, 6, c.max_blocks, window, 4) > 0
    verify(c, q, window, 4)
    c.close()


def test_single_tokens_match_the_decode_definition():
    n = np.array([1, 300, 77, 1000])
    c = case(n, [1] * 4, 32, 8, 128, 16, 100, 4)
    verify(c, c.normal(4, 32, 128), 100, 4)
    c.close()


@pytest.mark.parametrize("scale", [0.5, -0.3, 0.0])
def test_scales(scale):
    c = case([300], [200], 8, 2, 64, 16, 64, 4)
    verify(c, c.normal(c.T, 8, 64), 64, 4, scale=scale)
    c.close()


def test_many_short_chunks():
    rng = np.random.default_rng(2)
    nq = rng.integers(0, 9, 150)
    n = nq + rng.integers(0, 200, 150)
    c = case(n, nq, 8, 2, 64, 16, 60, 3, seed=8)
    verify(c, c.normal(c.T, 8, 64), 60, 3)
    verify(c, c.normal(c.T, 8, 64), 60, 3, max_q=c.T)  # any bound on the longest chunk
    c.close()


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_nan_and_infinities_reach_only_the_queries_that_see_them(window, sinks, bad):
    """A bad value in V of token 50 (one column of KV head 1) and of the last
    token (all of KV head 0)."""
    c = case([150], [150], 8, 2, 128, 16, window, sinks, seed=7, evict=False)
    b = c.host_table[0]
    c.pool[b[50 // 16], 1, 1, 50 % 16, 9] = bad
    c.pool[b[149 // 16], 1, 0, 149 % 16] = bad
    q = c.normal(c.T, 8, 128)
    ref, bound = c.reference(q, c.d ** -0.5, window, sinks)
    assert torch.isfinite(ref[:50]).all() and not torch.isfinite(ref[50, 4:, 9]).any()
    verify(c, q, window, sinks)
    c.close()


def test_nan_in_k_reaches_only_the_queries_that_see_it():
    c = case([140], [140], 4, 1, 64, 16, 30, 0, seed=7, evict=False)
    c.pool[c.host_table[0, 5], 0, 0, 2, 1] = float("nan")  # token 82
    q = c.normal(c.T, 4, 64)
    out = attend(c, q, 30, 0)
    bad = torch.isnan(out).all(-1).all(-1)
    assert bad.nonzero().flatten().tolist() == list(range(82, 112))
    assert torch.isfinite(out[~bad]).all()
    c.close()


def test_scores_of_the_lowest_values():
    """A score of -inf has weight 0 beside others, and alone its softmax is NaN;
    so has one that leaves fp32 (2 * -3e38): sums and scores are fp32."""
    from tests.paged_ref import check

    c = case([40], [40], 2, 1, 64, 16, 0, 0, seed=1)
    q = c.normal(40, 2, 64)
    q[:, :, 0] = 2.0
    c.pool[c.host_table[0, 0], 0, 0, 0] = 0
    c.pool[c.host_table[0, 0], 0, 0, 0, 0] = float("-inf")
    ref, bound = c.reference(q, 0.5, 0, 0)
    assert torch.isnan(ref[0]).all() and torch.isfinite(ref[1:]).all()
    check(attend(c, q, 0, 0, scale=0.5), ref, bound)
    c.pool[c.host_table[0, 0], 0, 0, 0, 0] = -3e38
    check(attend(c, q, 0, 0, scale=0.5), ref, bound)
    c.close()


def test_placement_does_not_change_bits():
    outs = []
    for spare in (3, 11):
        c = case([700, 300], [500, 33], 8, 2, 128, 16, 90, 4, seed=3, spare=spare)
        q = torch.randn(c.T, 8, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        outs.append(attend(c, q, 90, 4))
        c.close()
    assert torch.equal(outs[0], outs[1])


def test_another_stream():
    c = case([900], [700], 8, 2, 128, 16, 0, 0, seed=5)
    q = c.normal(c.T, 8, 128)
    want = attend(c, q, 0, 0)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    assert torch.equal(attend(c, q, 0, 0, stream=st), want)
    c.close()


def test_refusals_and_bounds():
    c = case([100, 5], [60, 5], 8, 2, 128, 16, 64, 4)
    q = c.normal(c.T, 8, 128)
    for kw in ({"window": -1}, {"sinks": -1}, {"scale": float("nan")}, {"max_q": c.T + 1}, {"max_q": 0}):
        with pytest.raises(K.KVError) as e:
            attend(c, q, kw.get("window", 64), kw.get("sinks", 4), scale=kw.get("scale"), max_q=kw.get("max_q"))
        assert e.value.code == K.KV_ERR_INVALID_ARG
    with pytest.raises(K.KVError) as e:
        K.kv_prompt_workspace_bytes(c.h, 0, 2, 12, 65, 60, c.max_blocks, 64, 4)  # 6 query heads a KV head
    assert e.value.code == K.KV_ERR_UNSUPPORTED
    # a length shorter than the chunk: the first queries see nothing
    c.lens[1] = 3
    out = attend(c, q, 64, 4)
    assert c.error() == K.KV_ERR_DEVICE_BOUNDS
    assert (out[60:62] == 0).all()
    c.lens[1] = 5
    # a block outside the pool is reported
    c.table[0, 5] = 10 ** 6
    attend(c, q, 64, 4)
    assert c.error() == K.KV_ERR_DEVICE_BOUNDS
    c.close()
    # nothing to do
    c = case([5], [0], 8, 2, 128, 16, 64, 4)
    K.paged_prompt_attn(c.h, 0, q, q, c.starts, 0, 0, c.table, c.lens, c.max_blocks, 1, 8, 1.0, 64, 4, None, 0)
    c.close()
