"""Normed rotary append against its definition in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


def expected(x, pos, freqs, rot, interleaved, weight, eps, offset, mag=1.0):
    """x [T, heads, d] float64 normed (weight None: not) and turned."""
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * (weight.double() + offset)
    ang = torch.from_numpy(np.asarray(pos, np.float64)[:, None] * freqs[None, :]).cuda()
    c, s = torch.cos(ang)[:, None] * mag, torch.sin(ang)[:, None] * mag
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def near(got, want):
    """One rounding to bf16, 2^-8 of the value; in fp32 before it the sum of d
    squares (2^-24 log2 d or less by pairs and shuffles, in all under 2^-20), its
    root (2^-22) and five products, of the larger of a pair: under 2^-18 of the
    row's largest."""
    tol = 2.0 ** -8 * want.abs() + 2.0 ** -18 * want.abs().amax(-1, keepdim=True) + 1e-30
    assert ((got.double() - want).abs() <= tol).all()


def verify(n, nq, Hq, Hkv, d, bs, rot, interleaved=False, eps=1e-6, offset=0.0, pad=0, which="qk", ragged=True,
           inplace=False, q=True, kv=True, positions=None, amp=3.0, stream=None):
    from tests.paged_ref import Paged

    c = Paged(n, nq, Hq, Hkv, d, bs, 11)
    freqs = K.kv_rotary_freqs(rot) if rot else np.zeros(0)
    rows = (c.normal(c.T, (Hq + 2 * Hkv) * d + pad).float() * amp).to(torch.bfloat16)
    xq, xk, xv = rows[:, : Hq * d], rows[:, Hq * d : (Hq + Hkv) * d], rows[:, (Hq + Hkv) * d : (Hq + 2 * Hkv) * d]
    if inplace:
        xq = xq.contiguous()
    wq, wk = (c.normal(d) if x in which else None for x in "qk")
    before = [t.reshape(c.T, -1, d).double() for t in (xq, xk, xv)]
    steps = torch.from_numpy(K.kv_rotary_steps(freqs).view(np.int64)).cuda() if rot else None
    R, N = K.Rotary(rot, steps, interleaved=interleaved), K.HeadNorm(wq, wk, eps, offset)
    out = xq if inplace else torch.full((c.T, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    pos_dev = None if positions is None else torch.from_numpy(positions.astype(np.int32)).cuda()
    pool0 = c.pool.clone()
    torch.cuda.synchronize()
    K.kv_append_rotary_norm(c.h, 0, R, N, xq if q else None, xq.stride(0), out if q else None, xk if kv else None,
                            xk.stride(0), xv if kv else None, xv.stride(0), pos_dev, c.starts if ragged else None, c.T,
                            c.table, c.lens, c.max_blocks, c.S, Hq, stream)
    torch.cuda.synchronize()
    seq = np.repeat(np.arange(c.S), c.nq)
    slot = (c.n - c.nq)[seq] + np.arange(c.T) - c.starts_host[seq]
    pos = slot if positions is None else positions
    if q:
        near(out.view(c.T, Hq, d), expected(before[0], pos, freqs, rot, interleaved, wq, eps, offset))
    if kv and c.T:
        b, o = (torch.from_numpy(t.astype(np.int64)).cuda() for t in (c.host_table[seq, slot // bs], slot % bs))
        got = c.pool[b, :, :, o]  # [T, 2, Hkv, d]
        near(got[:, 0], expected(before[1], pos, freqs, rot, interleaved, wk, eps, offset))
        assert torch.equal(got[:, 1].double(), before[2])
        pool0[b, :, :, o] = got
    assert torch.equal(c.pool.view(torch.int16), pool0.view(torch.int16))
    assert c.error() == 0
    c.close()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 16), (128, 128), (128, 64), (128, 48), (128, 0), (80, 32), (256, 256), (8, 0), (24, 16), (40, 32)])
@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (1, 1), (40, 8)])
def test_layouts(interleaved, d, rot, Hq, Hkv):
    verify([70, 3, 17, 16], [33, 3, 1, 16], Hq, Hkv, d, 16, rot, interleaved)


@pytest.mark.parametrize("bs", [1, 7, 16, 100])
def test_block_sizes_single_tokens_and_empty_chunks(bs):
    verify([9, 1, 300, 40], [0, 1, 1, 0], 8, 2, 128, bs, 128)


@pytest.mark.parametrize("kw", [
    {"ragged": False}, {"inplace": True}, {"q": False}, {"kv": False}, {"which": "q"}, {"which": "k"}, {"which": ""},
    {"offset": 1.0}, {"eps": 0.0}, {"eps": 0.5}, {"amp": 2.0 ** -50, "eps": 0.0}, {"amp": 2.0 ** 50}, {"pad": 24}])
def test_forms(kw):
    verify([9, 1, 300, 40], [1] * 4, 8, 2, 128, 16, 128, **{"pad": 8 if not kw.get("inplace") else 0, **kw})


@pytest.mark.parametrize("first", [0, 100000, 2**31 - 10, -70000])
def test_far_positions(first):
    verify([9, 5], [9, 5], 4, 2, 128, 16, 128, positions=first + np.minimum(np.arange(14), 9))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,rot", [(2, 1, 64, 64), (16, 4, 128, 128), (1, 1, 16, 16), (4, 1, 64, 32), (9, 3, 128, 48)])
def test_many_small_tokens(interleaved, Hq, Hkv, d, rot):
    """Groups of threads that share CTAs, some with a token more than others."""
    verify([4001, 37, 5000], [4001, 30, 3333], Hq, Hkv, d, 16, rot, interleaved)


def test_rows_of_zeros_and_not_numbers():
    """Zeros stay zeros with eps > 0; a NaN stays in its head."""
    from tests.paged_ref import Paged

    c = Paged([5], [5], 2, 1, 64, 16, 3)
    x = c.normal(5, 4 * 64).view(5, 4, 64)
    x[1, 0] = 0.0
    x[2, 1, 7] = float("nan")
    w = c.normal(64)
    steps = torch.from_numpy(K.kv_rotary_steps(K.kv_rotary_freqs(64)).view(np.int64)).cuda()
    out = torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    K.kv_append_rotary_norm(c.h, 0, K.Rotary(64, steps), K.HeadNorm(w, w), x, 256, out, x[:, 2], 256, x[:, 3], 256, None,
                            c.starts, 5, c.table, c.lens, c.max_blocks, 1, 2)
    torch.cuda.synchronize()
    assert (out[1, 0] == 0).all() and torch.isnan(out[2, 1]).all() and torch.isnan(out).sum() == 64
    c.close()


def test_another_stream_and_a_graph():
    from tests.paged_ref import Paged

    verify([70, 3], [33, 3], 8, 2, 128, 16, 128, stream=torch.cuda.Stream())
    c = Paged([70, 3], [1, 1], 8, 2, 128, 16, 3)
    x, w = c.normal(2, 12 * 128), c.normal(128)
    steps = torch.from_numpy(K.kv_rotary_steps(K.kv_rotary_freqs(128)).view(np.int64)).cuda()
    R, N = K.Rotary(128, steps), K.HeadNorm(w, w)
    outs = [torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def call(out, stream=None):
        K.kv_append_rotary_norm(c.h, 0, R, N, x, x.stride(0), out, x[:, 1024:], x.stride(0), x[:, 1280:], x.stride(0), None,
                                None, 2, c.table, c.lens, c.max_blocks, 2, 8, stream)

    call(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[1], torch.cuda.current_stream())
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and outs[0].abs().sum() > 0
    c.close()
