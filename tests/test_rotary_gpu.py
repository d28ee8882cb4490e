"""Rotary append against its definition in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


def rotated(x, pos, freqs, rot, interleaved, mag):
    """x [T, heads, d] float64 turned to positions pos."""
    T, H, d = x.shape
    ang = torch.from_numpy(np.asarray(pos, np.float64)[:, None] * freqs[None, :]).cuda()
    c, s = torch.cos(ang)[:, None] * mag, torch.sin(ang)[:, None] * mag
    y = x.clone()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        y[..., a] = x[..., a] * c[..., i] - x[..., b] * s[..., i]
        y[..., b] = x[..., b] * c[..., i] + x[..., a] * s[..., i]
    return y


def near(got, want, x):
    """One rounding to bf16 (2^-8 of the value), and fp32 products of the pair."""
    tol = 2.0 ** -8 * want.abs() + 2e-6 * x.abs().amax(-1, keepdim=True) + 1e-30
    assert ((got.double() - want).abs() <= tol).all()


def run(c, rot, freqs, interleaved=False, mag=1.0, pad=0, positions=None, ragged=True, q=True, kv=True, inplace=False):
    Hq, Hkv, d = c.Hq, c.Hkv, c.d
    rows = c.normal(c.T, (Hq + 2 * Hkv) * d + pad)
    xq, xk, xv = rows[:, : Hq * d], rows[:, Hq * d : (Hq + Hkv) * d], rows[:, (Hq + Hkv) * d : (Hq + 2 * Hkv) * d]
    if inplace:
        xq = xq.contiguous()
    before = [t.reshape(c.T, -1, d).double() for t in (xq, xk, xv)]
    steps = torch.from_numpy(K.kv_rotary_steps(freqs).view(np.int64)).cuda() if rot else None
    R = K.Rotary(rot, steps, interleaved=interleaved, magnitude=mag)
    out = xq if inplace else torch.full((c.T, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    pos_dev = None if positions is None else torch.from_numpy(positions.astype(np.int32)).cuda()
    K.kv_append_rotary(c.h, 0, R, xq if q else None, xq.stride(0), out if q else None, xk if kv else None,
                       xk.stride(0), xv if kv else None, xv.stride(0), pos_dev, c.starts if ragged else None, c.T,
                       c.table, c.lens, c.max_blocks, c.S, Hq)
    torch.cuda.synchronize()
    return before, out.view(c.T, Hq, d)


def verify(c, rot, freqs, **kw):
    pool0 = c.pool.clone()
    (q, k, v), out = run(c, rot, freqs, **kw)
    seq = np.repeat(np.arange(c.S), c.nq)
    slot = (c.n - c.nq)[seq] + np.arange(c.T) - c.starts_host[seq]
    pos = slot if kw.get("positions") is None else kw["positions"]
    inter, mag = kw.get("interleaved", False), kw.get("mag", 1.0)
    if kw.get("q", True):
        near(out, rotated(q, pos, freqs, rot, inter, mag), q)
        assert torch.equal(out[..., rot:].double(), q[..., rot:])
    if kw.get("kv", True):
        want = rotated(k, pos, freqs, rot, inter, mag)
        b, o = c.host_table[seq, slot // c.bs], slot % c.bs
        got = c.pool[torch.from_numpy(b.astype(np.int64)).cuda(), :, :, torch.from_numpy(o).cuda()]  # [T, 2, Hkv, d]
        near(got[:, 0], want, k)
        assert torch.equal(got[:, 1].double(), v)
        pool0[torch.from_numpy(b.astype(np.int64)).cuda(), :, :, torch.from_numpy(o).cuda()] = got
    # nothing else of the pool changed
    assert torch.equal(c.pool.view(torch.int16), pool0.view(torch.int16))
    assert c.error() == 0


def paged(n, nq, Hq, Hkv, d, bs, **kw):
    from tests.paged_ref import Paged

    return Paged(n, nq, Hq, Hkv, d, bs, 11, **kw)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 16), (128, 128), (128, 64), (128, 48), (128, 0), (80, 32), (256, 256)])
@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (1, 1), (40, 8)])
def test_layouts(interleaved, d, rot, Hq, Hkv):
    freqs = K.kv_rotary_freqs(rot) if rot else np.zeros(0)
    c = paged([70, 3, 17, 16], [33, 3, 1, 16], Hq, Hkv, d, 16)
    verify(c, rot, freqs, interleaved=interleaved)
    c.close()


@pytest.mark.parametrize("bs", [1, 7, 16, 100])
def test_block_sizes_single_tokens_and_empty_chunks(bs):
    c = paged([9, 1, 300, 40], [0, 1, 1, 0], 8, 2, 128, bs)
    verify(c, 128, K.kv_rotary_freqs(128))
    c.close()


def test_decode_form_and_strides():
    c = paged([9, 1, 300, 40], [1] * 4, 8, 2, 128, 16)
    verify(c, 128, K.kv_rotary_freqs(128), ragged=False, pad=24)
    verify(c, 128, K.kv_rotary_freqs(128), inplace=True)
    verify(c, 128, K.kv_rotary_freqs(128), q=False)
    verify(c, 128, K.kv_rotary_freqs(128), kv=False)
    c.close()


@pytest.mark.parametrize("first", [0, 100000, 2**31 - 10, -70000])
def test_far_positions(first):
    """The fraction of a turn is exact wherever the token stands."""
    c = paged([9, 5], [9, 5], 4, 2, 128, 16)
    verify(c, 128, K.kv_rotary_freqs(128, base=500000.0), positions=first + np.minimum(np.arange(14), 9))
    c.close()


def test_scaled_frequencies():
    f = K.kv_rotary_freqs(64, base=500000.0, scaling=K.KV_ROTARY_BY_PARTS, factor=8.0, original_len=8192)
    c = paged([900, 70], [33, 60], 8, 2, 64, 32)
    verify(c, 64, f, interleaved=True, mag=1.2079)
    c.close()


def test_many_sequences():
    rng = np.random.default_rng(0)
    nq = rng.integers(0, 5, 1100)
    c = paged(nq + rng.integers(0, 60, 1100), nq, 2, 1, 64, 16)
    verify(c, 64, K.kv_rotary_freqs(64))
    c.close()


def test_bounds_are_reported_and_skipped():
    c = paged([40, 20], [4, 4], 4, 2, 64, 16)
    before = c.pool.clone()
    c.lens[0] = 2           # two of four tokens before position 0
    c.table[1, 1] = 10 ** 6  # outside the pool
    run(c, 64, K.kv_rotary_freqs(64))
    assert c.error() == K.KV_ERR_DEVICE_BOUNDS
    changed = (c.pool.view(torch.int16) != before.view(torch.int16)).flatten(1).any(1).nonzero().flatten().tolist()
    assert changed == [int(c.host_table[0, 0])]  # the two tokens at positions 0 and 1
    c.lens[:] = 0            # no context: nothing is written, nothing reported
    before = c.pool.clone()
    run(c, 64, K.kv_rotary_freqs(64))
    assert c.error() == 0 and torch.equal(c.pool.view(torch.int16), before.view(torch.int16))
    c.close()


def test_refusals():
    c = paged([40], [4], 4, 2, 64, 16)
    f = K.kv_rotary_freqs(64)
    steps = torch.from_numpy(K.kv_rotary_steps(f).view(np.int64)).cuda()
    q, k = c.normal(4, 4 * 64), c.normal(4, 2 * 64)
    ok = dict(q=q, qs=256, o=torch.empty_like(q), k=k, ks=128, v=k, vs=128, T=4, S=1, rot=64, mag=1.0, st=steps)

    def call(**kw):
        a = {**ok, **kw}
        K.kv_append_rotary(c.h, 0, K.Rotary(a["rot"], a["st"], magnitude=a["mag"]), a["q"], a["qs"], a["o"], a["k"],
                           a["ks"], a["v"], a["vs"], None, c.starts, a["T"], c.table, c.lens, c.max_blocks, a["S"], 4)

    call()
    for bad in ({"qs": 248}, {"qs": 260}, {"ks": 120}, {"vs": 129}, {"q": q.data_ptr() + 2}, {"o": None}, {"v": None},
                {"T": -1}, {"rot": 80}, {"rot": -16}, {"mag": float("nan")}, {"st": None}, {"o": q, "qs": 512},
                {"q": None, "k": None, "v": None}):
        with pytest.raises(K.KVError) as e:
            call(**bad)
        assert e.value.code == K.KV_ERR_INVALID_ARG, bad
    with pytest.raises(K.KVError) as e:
        call(rot=24)
    assert e.value.code == K.KV_ERR_UNSUPPORTED
    c.close()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,rot", [(2, 1, 64, 64), (16, 4, 64, 32), (8, 2, 128, 128), (1, 1, 128, 48), (5, 1, 256, 0),
                                          (40, 8, 128, 64)])
@pytest.mark.parametrize("T", [1000, 2000, 7001])
def test_runs_of_tokens(T, Hq, Hkv, d, rot, interleaved):
    """Many tokens: small ones share CTAs, each group of threads takes a run of
    them, over the ends of sequences and over sequences without new tokens."""
    rng = np.random.default_rng(T)
    nq = rng.integers(0, 40, T)
    nq[5:9] = 0
    nq = nq[: int(np.searchsorted(np.cumsum(nq), T)) + 1]
    nq[-1] -= nq.sum() - T
    c = paged(nq + rng.integers(0, 50, len(nq)), nq, Hq, Hkv, d, 16)
    assert c.T == T
    verify(c, rot, K.kv_rotary_freqs(rot) if rot else np.zeros(0), interleaved=interleaved)
    c.close()


def test_runs_of_single_tokens():
    rng = np.random.default_rng(5)
    c = paged(rng.integers(1, 60, 4001), [1] * 4001, 4, 2, 64, 16)
    verify(c, 64, K.kv_rotary_freqs(64), ragged=False, pad=8)
    verify(c, 64, K.kv_rotary_freqs(64), ragged=False, q=False)
    verify(c, 64, K.kv_rotary_freqs(64), kv=False, positions=rng.integers(-9, 10 ** 6, 4001))
    c.close()


def test_bounds_within_runs():
    c = paged([20] * 1000, [4] * 1000, 4, 2, 64, 16)  # the new tokens at 16 .. 19
    before = c.pool.clone()
    c.lens[10:20] = 0          # no context: nothing is written
    c.lens[30:40] = 2          # two of four tokens before position 0
    c.table[50:60, 1] = -1     # no block
    c.table[70:80, 1] = 10 ** 6
    run(c, 64, K.kv_rotary_freqs(64))
    assert c.error() == K.KV_ERR_DEVICE_BOUNDS
    changed = (c.pool.view(torch.int16) != before.view(torch.int16)).flatten(1).any(1).nonzero().flatten().tolist()
    want = {int(c.host_table[s, 1]) for s in range(1000) if not any(a <= s < a + 10 for a in (10, 30, 50, 70))}
    assert set(changed) == want | {int(c.host_table[s, 0]) for s in range(30, 40)}
    c.close()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,rot", [(2, 1, 64, 64), (5, 1, 64, 32), (1, 1, 128, 128), (1, 1, 128, 48), (3, 1, 80, 16)])
@pytest.mark.parametrize("T", [8000, 15013])
def test_groups_below_a_warp(T, Hq, Hkv, d, rot, interleaved):
    """So many small tokens that a warp's threads are two or four tokens'."""
    rng = np.random.default_rng(T)
    nq = rng.integers(0, 90, T)
    nq[3:8] = 0
    nq = nq[: int(np.searchsorted(np.cumsum(nq), T)) + 1]
    nq[-1] -= nq.sum() - T
    c = paged(nq + rng.integers(0, 50, len(nq)), nq, Hq, Hkv, d, 16)
    assert c.T == T
    verify(c, rot, K.kv_rotary_freqs(rot), interleaved=interleaved, pad=8)
    c.close()


def test_groups_below_a_warp_single_tokens_and_bounds():
    rng = np.random.default_rng(6)
    c = paged(rng.integers(1, 40, 15000), [1] * 15000, 2, 1, 64, 16)
    verify(c, 64, K.kv_rotary_freqs(64), ragged=False)
    verify(c, 64, K.kv_rotary_freqs(64), q=False)
    before = c.pool.clone()
    c.lens[100:111] = 0       # no context: nothing is written
    c.table[200:213] = -1     # no block
    run(c, 64, K.kv_rotary_freqs(64))
    assert c.error() == K.KV_ERR_DEVICE_BOUNDS
    changed = (c.pool.view(torch.int16) != before.view(torch.int16)).flatten(1).any(1).nonzero().flatten().tolist()
    want = {int(c.host_table[s, (c.n[s] - 1) // 16]) for s in range(15000) if not (100 <= s < 111 or 200 <= s < 213)}
    assert set(changed) == want
    c.close()
