"""The packed layer as it is used: chunked prompts, forks, decode steps that pack
the pages they fill, releases, compaction, streams.  The cache is read back byte by
byte: its rows against the definition of the append and of packing, and each
output against attention in 64 bits over what the cache held."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


class Chats:
    """A layer's slots: every token's normed and turned k and its v in 64 bits, and
    the cache's own rows as they stand."""

    def __init__(self, layer, freqs, wq, wk, eps):
        self.layer, self.f, self.wq, self.wk, self.eps = layer, torch.from_numpy(freqs).cuda(), wq, wk, eps
        S, Hkv, d = layer.S, layer.Hkv, layer.d
        self.k = [torch.zeros(0, Hkv, d, dtype=torch.float64, device="cuda") for _ in range(S)]
        self.v = [torch.zeros(0, Hkv, d, dtype=torch.float64, device="cuda") for _ in range(S)]

    def turned(self, x, heads, w, first):  # half layout
        x = x.double().view(len(x), heads, -1)
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + self.eps) * w.double()
        ang = torch.arange(first, first + len(x), device="cuda").double().view(-1, 1, 1) * self.f
        r = len(self.f)
        a, b = x[..., :r], x[..., r : 2 * r]
        return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin(), x[..., 2 * r :]], -1)

    def cache(self, s):
        """Slot s's rows [2, Hkv, n, d] in 64 bits, each one's greatest possible
        distance from the row that was appended, and the tokens in 4 bits."""
        from tests.q4_ref import parse_block

        L = self.layer
        torch.cuda.synchronize()
        (t, n), (t4, n4) = L.tab.host(), L.tab4.host()
        n, p, page = int(n[s]), int(n4[s]), L.Hkv * L.bs * L.d // 8
        rows, off = [torch.zeros(2, L.Hkv, 0, L.d, dtype=torch.float64, device="cuda")], []
        for j in range(p // L.bs):
            raw = L.pool.buf[int(t4[s, j]) * page :][: 9 * page].cpu().numpy()
            c, sc, z = (torch.from_numpy(x).cuda().double() for x in parse_block(raw, L.Hkv, L.bs, L.d))
            rows.append((c * sc + z).flatten(-2))
            # half a step, s = bf16(span / 15): the last code is 2^-8 of the span short at most
            off.append((0.5 * sc + 15 * sc * 2.0 ** -7).expand(*sc.shape[:-1], 64).flatten(-2))
        for j in range(p // L.bs, -(-n // L.bs)):
            b = L.pool.buf[int(t[s, j]) * page :][: 32 * page].view(torch.bfloat16).view(2, L.Hkv, L.bs, L.d)
            rows.append(b[:, :, : n - j * L.bs].double())
            off.append(torch.zeros_like(rows[-1]))
        return torch.cat(rows, 2), (torch.cat(off, 2) if off else rows[0]), p

    def check_cache(self, s):
        rows, off, p = self.cache(s)
        for got, far, want in ((rows[0], off[0], self.k[s]), (rows[1], off[1], self.v[s])):
            want = want.transpose(0, 1)
            # the append's rounding (2^-8) and fp32 sums (2^-18 of the row), then packing
            tol = 2.0 ** -8 * want.abs() + 2.0 ** -18 * want.abs().amax(-1, keepdim=True) + 1e-9
            assert ((got - want).abs() <= tol + far).all()

    def expect(self, s, q, k, v):
        """New rows of slot s; what attention gives over the cache as it stands with
        the new rows behind it, and the sums of weight * |v|."""
        L, n0, n = self.layer, len(self.k[s]), len(q)
        old = self.cache(s)[0]
        q, k, v = self.turned(q, L.Hq, self.wq, n0), self.turned(k, L.Hkv, self.wk, n0), v.double().view(n, L.Hkv, L.d)
        self.k[s], self.v[s] = torch.cat([self.k[s], k]), torch.cat([self.v[s], v])
        b = lambda x: x.float().to(torch.bfloat16).double()  # noqa: E731
        keys, values = torch.cat([old[0], b(k).transpose(0, 1)], 1), torch.cat([old[1], v.transpose(0, 1)], 1)
        hidden = torch.arange(n0 + n, device="cuda") > torch.arange(n0, n0 + n, device="cuda").view(-1, 1)
        w = torch.einsum("nhgd,hjd->hgnj", b(q).view(n, L.Hkv, -1, L.d), keys) * L.scale
        w = torch.softmax(w.masked_fill(hidden, -np.inf), -1)
        o, a = (torch.einsum("hgnj,hjd->nhgd", w, x).reshape(n, L.Hq, L.d) for x in (values, values.abs()))
        return o, a


def near(got, want, bound, unpacked=0.0):
    # output and weights rounded to bf16 at most (2^-8 each); a rounding of q or k that
    # falls the other way moves a score by 2^-8 of a product of two columns: taken as 2%
    # of the weights, as over windows; a prompt reads packed rows rounded to bf16 once
    # more: every product of a score 2^-8 off at most, and V's columns
    tol = 2.0 ** -8 * 1.02 * (want.abs() + bound) + (0.02 + unpacked) * bound + 1e-6
    assert ((got.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("d,bs,keep", [(128, 16, 20), (64, 32, 1)])
def test_chats_as_they_are_used(d, bs, keep):
    from paper_2606_12950_gb300.streaming import PackedLayer

    S, Hq, Hkv, eps = 5, 8, 2, 1e-5
    g = torch.Generator(device="cuda")
    g.manual_seed(d)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)

    freqs = K.kv_rotary_freqs(d)
    wq, wk = (1 + 0.3 * normal(2, d).float()).to(torch.bfloat16)
    layer = PackedLayer(90, Hq, Hkv, d, bs, S, 700, keep, freqs, norm=K.HeadNorm(wq, wk, eps))
    chats = Chats(layer, freqs, wq, wk, eps)

    def rows(n):
        x = normal(n, (Hq + 2 * Hkv) * d)
        return x[:, : Hq * d], x[:, Hq * d : (Hq + Hkv) * d], x[:, (Hq + Hkv) * d :]

    def prompt(counts, stream=None):
        q, k, v = rows(sum(counts))
        at, want = 0, []
        again = [bool(layer.tab4.lens()[s]) for s in range(S)]
        for s, n in enumerate(counts):
            if n:
                want.append((slice(at, at + n), *chats.expect(s, q[at : at + n], k[at : at + n], v[at : at + n]), again[s]))
            at += n
        out = layer.prompt(counts, q, k, v, stream)
        torch.cuda.synchronize()
        for where, o, a, was_packed in want:
            near(out[where], o, a, 0.02 if was_packed else 0.0)

    def step(stream=None):
        live = np.nonzero(layer.tab.lens())[0]
        q, k, v = rows(S)
        want = {s: chats.expect(s, q[s : s + 1], k[s : s + 1], v[s : s + 1]) for s in live}
        out = layer.step(q, k, v, stream)
        torch.cuda.synchronize()
        for s in range(S):
            if s in want:
                near(out[s : s + 1], *want[s])
            else:
                assert (out[s] == 0).all()

    def invariant():
        n, p = layer.tab.lens(), layer.tab4.lens()
        assert (p == np.maximum(0, n - keep) // bs * bs).all()
        table, table4 = layer.tab.host()[0], layer.tab4.host()[0]
        for s in range(S):
            b = p[s] // bs
            assert (table[s, :b] == -1).all() and (table4[s, :b] >= 0).all() and (table[s, b : -(-n[s] // bs)] >= 0).all()
            chats.check_cache(s)

    prompt([150, 3, 0, bs + keep, 0])
    invariant()
    for _ in range(bs + 3):
        step()
    invariant()
    layer.fork(0, [2, 4])
    for s in (2, 4):
        chats.k[s], chats.v[s] = chats.k[0], chats.v[0]
    held = layer.packed_used()
    assert held == sum(int(x) // bs for x in layer.tab4.lens()[[0, 1, 3]])  # forks share
    prompt([0, 60, 37, 0, 0])     # a chat with packed pages, forked, goes on
    invariant()
    other = torch.cuda.Stream()
    for i in range(bs + 2):
        step(other if i % 2 else None)
    invariant()
    layer.release(0)
    chats.k[0], chats.v[0] = chats.k[0][:0], chats.v[0][:0]
    layer.release(3)
    chats.k[3], chats.v[3] = chats.k[3][:0], chats.v[3][:0]
    moved = layer.compact()
    invariant()
    step()
    prompt([70, 1, 0, 5, 9])
    invariant()
    assert moved > 0
    assert layer.pool.error() == 0
    layer.close()


def test_no_room_for_packing_or_copies():
    """Without a page for packing the tokens stay in bf16; with one, a few pages are
    packed at a time; a prompt that needs copies the pool has no pages for is refused
    with nothing changed."""
    from paper_2606_12950_gb300.streaming import PackedLayer

    d, bs, S, Hq, Hkv = 64, 16, 2, 2, 2
    layer = PackedLayer(8, Hq, Hkv, d, bs, S, 200, 1, K.kv_rotary_freqs(d))
    x = lambda n: torch.randn(n, 6 * d, device="cuda").to(torch.bfloat16)  # noqa: E731
    cut = lambda y: (y[:, : 2 * d], y[:, 2 * d : 4 * d], y[:, 4 * d :])  # noqa: E731
    layer.prompt([128, 0], *cut(x(128)))       # every page in bf16: none to pack into
    assert layer.tab4.lens()[0] == 0 and layer.pages_used() == 8
    layer.release(0)
    layer.prompt([100, 0], *cut(x(100)))       # seven pages; six of them packed, three at first
    assert layer.packed_used() == 6 and layer.pages_used() == 1 and layer.tab4.lens()[0] == 96
    K.kv_pool_trim(layer.pool.handle)
    hog = K.kv_alloc_blocks(layer.pool.handle, 0, 3)
    with pytest.raises(K.KVError) as e:
        layer.prompt([20, 0], *cut(x(20)))     # one more page, and six for copies, of two
    assert e.value.code == K.KV_ERR_OUT_OF_BLOCKS
    assert layer.tab.lens()[0] == 100 and layer.tab4.lens()[0] == 96 and layer.packed_used() == 6
    K.kv_free_blocks(layer.pool.handle, 0, hog)
    with pytest.raises(K.KVError):
        layer.prompt([20, 0], *cut(x(20)))     # of five
    layer.release(0)
    layer.prompt([60, 0], *cut(x(60)))         # three packed pages
    out = layer.prompt([20, 0], *cut(x(20)))   # their copies are given back
    torch.cuda.synchronize()
    assert torch.isfinite(out).all() and layer.pool.error() == 0
    assert layer.tab4.lens()[0] == 64 and layer.pages_used() == 1
    layer.close()


def test_arguments_and_empty_calls():
    from paper_2606_12950_gb300.streaming import PackedLayer

    f = K.kv_rotary_freqs(64)
    with pytest.raises(ValueError):
        PackedLayer(8, 2, 2, 64, 16, 2, 200, 0, f)
    layer = PackedLayer(8, 2, 2, 64, 16, 2, 200, 5, f)
    x = torch.randn(2, 6 * 64, device="cuda").to(torch.bfloat16)
    q, k, v = x[:, :128], x[:, 128:256], x[:, 256:]
    assert layer.prompt([0, 0], q[:0], k[:0], v[:0]).shape == (0, 2, 64)
    assert (layer.step(q, k, v) == 0).all()
    for bad in ((q.float(), k, v), (q, k[:1], v), (q, k, v[:, 1:])):
        with pytest.raises(ValueError):
            layer.step(*bad)
        with pytest.raises(ValueError):
            layer.prompt([1, 1], *bad)
    assert layer.tab.lens().sum() == 0
    layer.close()
