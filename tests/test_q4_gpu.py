"""Blocks packed into 4 bits against their definition, and decode attention over
them against 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


def ref():
    from tests import q4_ref

    return q4_ref


class Blocks:
    """n bf16 blocks of given values, n packed ones, n more bf16 ones."""

    def __init__(self, x):
        n, _, Hkv, bs, d = x.shape
        self.shape, self.block = (Hkv, bs, d), 2 * Hkv * bs * d * 2
        self.buf = torch.zeros((2 * n + -(-n // 3) + 1) * self.block, dtype=torch.uint8, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.h = K.kv_pool_create(self.buf, self.buf.numel(), bs, [(Hkv, d), (Hkv, d | K.KV_Q4)], self.err,
                                  page_bytes=self.block // 32, shuffle_seed=3)
        self.a, self.b = K.kv_alloc_blocks(self.h, 0, n), K.kv_alloc_blocks(self.h, 0, n)
        self.q = K.kv_alloc_blocks(self.h, 1, n)
        for i, v in zip(self.a, x):
            self.at(i)[:] = v

    def at(self, i):
        Hkv, bs, d = self.shape
        return self.buf[int(i) * self.block // 32 :][: self.block].view(torch.bfloat16).view(2, Hkv, bs, d)

    def parsed(self, i):
        torch.cuda.synchronize()
        return ref().parse_block(self.buf[int(i) * self.block // 32 :][: self.block * 9 // 32].cpu().numpy(), *self.shape)

    def close(self):
        torch.cuda.synchronize()
        K.kv_pool_destroy(self.h)


def normal(*shape, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def verify_blocks(x):
    b = Blocks(x)
    K.kv_pack_blocks(b.h, 0, 1, b.a, b.q)
    K.kv_unpack_blocks(b.h, 1, 0, b.q, b.b)
    torch.cuda.synchronize()
    for i, (p, u) in enumerate(zip(b.q, b.b)):
        c, s, z = ref().quantised(x[i])
        got_c, got_s, got_z = (torch.from_numpy(t).cuda() for t in b.parsed(p))
        assert torch.equal(torch.isnan(got_s), torch.isnan(s))
        ok = ~torch.isnan(s)
        assert torch.equal(got_s[ok], s[ok]) and torch.equal(got_z[ok], z[ok])
        assert torch.equal(got_c.double() * ok, c * ok)
        want = (c.float() * s + z).flatten(-2).to(torch.bfloat16)  # exact products, one fp32 sum
        got = b.at(u)
        nan = torch.isnan(want)
        assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])
        assert torch.equal(b.at(b.a[i]).view(torch.int16), x[i].view(torch.int16))
    b.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hkv,bs", [(2, 16), (1, 32), (3, 48), (8, 64), (2, 256), (16, 16)])
def test_pack_and_unpack(Hkv, bs, d):
    verify_blocks((normal(5, 2, Hkv, bs, d, seed=bs) * 3).to(torch.bfloat16))


def test_pack_odd_values():
    """Constant rows, halves of codes, huge and tiny spans, infinities, NaN."""
    x = normal(4, 2, 2, 16, 128, seed=4).to(torch.bfloat16)
    x[0, 0, 0, 0] = 0.0
    x[0, 0, 0, 1] = -0.0
    x[0, :, 0, 2] = 7.25
    x[0, :, 0, 3, ::2] = 3.0e38
    x[0, :, 0, 4, 5] = float("inf")
    x[0, :, 0, 5, 70] = float("-inf")
    x[0, :, 0, 6, 64:] = float("nan")
    x[0, :, 0, 7, 3] = float("nan")
    x[0, :, 0, 8] *= 2.0 ** -100
    x[0, :, 0, 9] *= 2.0 ** -128
    x[0, :, 0, 10] *= 2.0 ** 77
    x[0, :, 0, 11] *= 2.0 ** 90
    x[0, :, 0, 12] = x[0, :, 0, 12] * 0.001 + 1000.0
    x[0, :, 0, 13, 0] = 1.0e30  # the group's others lose themselves in its span
    x[1] = torch.randint(0, 31, x[1].shape, device="cuda") * 0.5  # s = 1: halves of codes
    x[1, ..., 0], x[1, ..., 1], x[1, ..., 64], x[1, ..., 65] = 0.0, 15.0, 0.0, 15.0
    x[2] = torch.randint(0, 121, x[2].shape, device="cuda") * 0.125
    verify_blocks(x)


@pytest.mark.parametrize("n", [1, 119, 121, 505, 2050])
def test_pack_many_blocks(n):
    """Over each size of a launch's parameters; and a block packed twice."""
    x = normal(n, 2, 2, 16, 64, seed=n).to(torch.bfloat16)
    b = Blocks(x)
    K.kv_pack_blocks(b.h, 0, 1, b.a, b.q)
    K.kv_unpack_blocks(b.h, 1, 0, b.q, b.b)
    c, s, z = ref().quantised(x)
    want = (c.float() * s + z).flatten(-2).to(torch.bfloat16)
    torch.cuda.synchronize()
    for i in range(n):
        assert torch.equal(b.at(b.b[i]), want[i])
    if n > 1:
        K.kv_pack_blocks(b.h, 0, 1, [b.a[1], b.a[1]], [b.q[0], b.q[1]])
        torch.cuda.synchronize()
        assert np.array_equal(b.parsed(b.q[0])[0], b.parsed(b.q[1])[0])
    b.close()


def attend(n, p, Hq, Hkv, d, bs, seed=5, scale=None, q=None, **kw):
    c = ref().PagedQ4(n, p, Hq, Hkv, d, bs, seed, **kw)
    q = c.normal(c.S, Hq, d) if q is None else q
    scale = d ** -0.5 if scale is None else scale
    out = c.run(q, scale)
    torch.cuda.synchronize()
    ref().check(out, *c.reference(q, scale))
    assert c.error() == 0
    return c, q, out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (4, 2), (8, 2), (10, 2), (16, 2), (40, 8), (3, 3)])
def test_heads(Hq, Hkv, d):
    attend([70, 1, 300, 33, 160], [48, 0, 272, 32, 144], Hq, Hkv, d, 16)[0].close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bs", [16, 32, 48, 64, 256])
@pytest.mark.parametrize("append", [True, False])
def test_lengths(bs, d, append):
    """Empty, one token, block edges, all or nothing in 4 bits."""
    n, p = [], []
    for m in (0, 1, 2, bs - 1, bs, bs + 1, 2 * bs, 3 * bs + 7, 6 * bs + 1):
        for k in {0, m // bs * bs, (m - 1) // bs * bs, m // bs // 2 * bs}:
            if 0 <= k <= m - (append and m > 0):
                n.append(m)
                p.append(k)
    attend(n, p, 8, 2, d, bs, append=append)[0].close()


def test_the_new_row_is_appended():
    c = ref().PagedQ4([17, 48, 100, 0], [16, 32, 96, 0], 8, 2, 128, 16, 3)
    before = c.buf.clone()
    c.run(c.normal(4, 8, 128), 0.09)
    torch.cuda.synchronize()
    for s, n in enumerate([17, 48, 100]):
        b = c.block16(c.host_table[s, (n - 1) // 16])
        assert torch.equal(b[0, :, (n - 1) % 16], c.k_new[s]) and torch.equal(b[1, :, (n - 1) % 16], c.v_new[s])
        b[:, :, (n - 1) % 16] = before[int(c.host_table[s, (n - 1) // 16]) * c.block // 32 :][: c.block].view(
            torch.bfloat16).view(2, 2, 16, 128)[:, :, (n - 1) % 16]
    assert torch.equal(before, c.buf)  # nothing else
    c.close()


def test_many_sequences():
    """More than a CTA's threads, of all lengths and shares."""
    rng = np.random.default_rng(2)
    n = rng.integers(0, 400, 700)
    n[rng.integers(0, 700, 60)] = 0
    p = (rng.integers(0, 17, 700) * n // 16 - 1).clip(0) // 16 * 16
    c, q, out = attend(n, p, 4, 2, 64, 16)
    assert (out[torch.from_numpy(n == 0).cuda()] == 0).all()
    c.close()


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 8, 2), (64, 5, 1)])
def test_one_long_context(d, Hq, Hkv):
    attend([30011], [29952], Hq, Hkv, d, 64)[0].close()


def test_long_and_short_together():
    attend([20000, 3, 65, 9000, 16], [19968, 0, 48, 0, 0], 16, 4, 128, 16)[0].close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["two", "among short ones", "none", "one token"])
def test_many_runs(kind, d):
    """So many runs that the merge goes by parts, not by runs: all but two empty
    (fewer parts than there are CTAs, a run over most of them), a long one among
    short ones, none with a token."""
    n, p = np.zeros(320, np.int64), np.zeros(320, np.int64)
    if kind == "two":
        n[100], p[100], n[319], p[319] = 20007, 19984, 5, 0
    elif kind == "among short ones":
        n[:] = np.arange(320) % 45
        p[:] = (n - 1).clip(0) // 16 * 16
        n[160], p[160] = 30011, 29984
    elif kind == "one token":
        n[7] = 1
    c, q, out = attend(n, p, 8, 4, d, 16)
    assert (out[torch.from_numpy(n == 0).cuda()] == 0).all()
    assert torch.equal(c.run(q, d ** -0.5), out)
    c.close()


@pytest.mark.parametrize("append", [True, False])
def test_scales_far_apart(append):
    """Rows of V whose scales differ by many powers of two, within a tile, from
    tile to tile and from sequence to sequence; sharp and flat weights."""
    def make(kv, s, m):
        x = torch.randn(2, m, 128, device="cuda", generator=gen)
        if kv == 1:
            e = torch.randint(-30, 31, (m,), device="cuda", generator=gen).float()
            step = (torch.arange(m, device="cuda") // 64 % 5 - 2) * 20.0
            x = x * torch.exp2([e, step, torch.zeros_like(e) + 40, torch.zeros_like(e) - 50, e * 0][s % 5])[None, :, None]
            if s == 4:
                x = x * 0 + 3.5  # every scale 0
        return x.to(torch.bfloat16)

    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    n = [700, 701, 333, 330, 300]
    for scale in (0.02, 0.5):
        c = ref().PagedQ4(n, [640, 688, 320, 320, 288], 8, 2, 128, 16, 4, append=append, make=make)
        q = c.normal(5, 8, 128)
        out = c.run(q, scale)
        torch.cuda.synchronize()
        want, tol = c.reference(q, scale)
        # weights under 2^-22 of the largest lose bits in fp16: 2^-25 of 2^15 over it,
        # times the largest scale seen with them
        big = torch.stack([x[1].double().abs().amax() if x.shape[2] else x.new_zeros(()).double() for x in c.rows])
        ref().check(out, want, tol + 2.0 ** -21 * big.view(-1, 1, 1))
        c.close()


@pytest.mark.parametrize("mag", [2.0 ** -60, 2.0 ** -20, 2.0 ** 20, 2.0 ** 60])
def test_magnitudes_of_q_and_k(mag):
    """The same scores from q and k of any magnitude."""
    c = ref().PagedQ4([200, 90], [176, 64], 8, 2, 128, 16, 6,
                      make=lambda kv, s, m: (torch.randn(2, m, 128, device="cuda", generator=gen(s, kv)) *
                                             (1 / mag if kv == 0 else 1)).to(torch.bfloat16))
    q = (c.normal(2, 8, 128).float() * mag).to(torch.bfloat16)
    out = c.run(q, 128 ** -0.5)
    torch.cuda.synchronize()
    ref().check(out, *c.reference(q, 128 ** -0.5))
    c.close()


def gen(s, kv):
    g = torch.Generator(device="cuda")
    g.manual_seed(10 * s + kv)
    return g


@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0])
def test_other_scales(scale):
    # (scale 3: the scores' terms add to 128 times as much, and so does their error)
    c = ref().PagedQ4([200, 90, 40], [176, 64, 16], 8, 2, 64, 16, 6)
    q = c.normal(3, 8, 64)
    out = c.run(q, scale)
    torch.cuda.synchronize()
    want, tol = c.reference(q, scale)
    mag = torch.stack([x[1].double().abs().amax() for x in c.rows]).view(-1, 1, 1)
    ref().check(out, want, tol + (2.0 ** -9 * mag if scale == 3.0 else 0.0))
    c.close()


def test_not_numbers_stay_where_they_are():
    """A NaN in V reaches its group's columns, one in K or q the whole row."""
    def make(kv, s, m):
        x = torch.randn(2, m, 128, device="cuda", generator=gen(s, kv))
        if s == 0 and kv == 1:
            x[0, 5, 70] = float("nan")     # packed: columns 64 and on of head 0
        if s == 1 and kv == 0:
            x[1, 20, 3] = float("inf")     # packed
        if s == 2 and kv == 1:
            x[1, 45, 3] = float("nan")     # bf16: that column
        return x.to(torch.bfloat16)

    c = ref().PagedQ4([50, 50, 50, 50], [32, 32, 32, 32], 8, 2, 128, 16, 6, make=make)
    q = c.normal(4, 8, 128)
    q[3, 2, 9] = float("nan")
    out = c.run(q, 0.09)
    torch.cuda.synchronize()
    nan = torch.zeros(4, 8, 128, dtype=torch.bool, device="cuda")
    nan[0, :4, 64:] = nan[1, 4:] = nan[2, 4:, 3] = nan[3, 2] = True
    assert torch.equal(torch.isnan(out), nan)
    assert c.error() == 0
    c.close()


def test_results_do_not_depend_on_places_streams_or_graphs():
    outs = []
    n, p = [900, 77, 400, 31], [864, 64, 0, 16]
    for seed in (1, 2):  # other blocks, the same rows
        c = ref().PagedQ4(n, p, 16, 4, 128, 16, seed,
                          make=lambda kv, s, m: torch.randn(4, m, 128, device="cuda", generator=gen(s, kv)).to(torch.bfloat16))
        q = torch.randn(4, 16, 128, device="cuda", generator=gen(9, 9)).to(torch.bfloat16)
        outs.append(c.run(q, 0.09))
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        outs.append(c.run(q, 0.09, stream=st))
        torch.cuda.synchronize()
        out, graph = torch.zeros_like(outs[0]), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run(q, 0.09, out=out, stream=torch.cuda.current_stream())
        out.fill_(7.0)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        outs.append(out.clone())
        c.close()
    for o in outs[1:]:
        assert torch.equal(o, outs[0])


def test_bad_lengths_and_entries_set_the_error_word():
    """What the kernel's own checks turn away: no access, the word set."""
    for change in ("packed past the length", "packed odd", "length past the table", "negative", "entry", "entry4", "no room"):
        c = ref().PagedQ4([100, 60], [80, 32], 8, 2, 128, 16, 3)
        if change == "packed past the length":
            c.packed[0] = 112
        elif change == "packed odd":
            c.packed[0] = 72
        elif change == "length past the table":
            c.lens[0] = 100000
        elif change == "negative":
            c.lens[0] = -5
        elif change == "entry":
            c.table[0, 5] = 1 << 29
        elif change == "entry4":
            c.table4[0, 2] = -1
        else:
            c.lens[0], c.packed[0] = 80, 80  # all in 4 bits: no place for the new row
        q = c.normal(2, 8, 128)
        out = c.run(q, 0.09)
        torch.cuda.synchronize()
        assert c.error() == K.KV_ERR_DEVICE_BOUNDS, change
        want, tol = c.reference(q, 0.09)
        ref().check(out[1], want[1], tol[1])  # the other sequence is as ever
        c.close()


@pytest.mark.parametrize("d,n", [(64, 16400), (128, 16400)])
def test_long_runs_in_one_warp_do_not_drift(d, n):
    """As many contexts as warps, so that a warp takes each from end to end, with
    nearly flat weights: the output is small beside what its sums are made of.  (All
    read the same blocks.)  Rounding moves the output by 2^-8 of its norm at most,
    and weights off by 2^-11 each, on their own, by 2^-11 sum(p s c) / sqrt(n) a
    column: under 2^-9 of a mean of n values about as large."""
    c = ref().PagedQ4([n], [n // 16 * 16 - 16], 1, 1, d, 16, 5, append=False)
    S = 2560
    table, table4 = c.table.expand(S, -1).contiguous(), c.table4.expand(S, -1).contiguous()
    lens, packed = c.lens.expand(S).contiguous(), c.packed.expand(S).contiguous()
    q = (c.normal(S, 1, d).float() * 0.05).to(torch.bfloat16)
    out = torch.empty(S, 1, d, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(K.kv_q4_workspace_bytes(c.h, 1, S, 1, c.max_blocks), dtype=torch.uint8, device="cuda")
    K.paged_decode_attn_q4(c.h, 0, 1, q, None, None, out, table, lens, c.max_blocks, table4, packed, c.max_blocks4, S, 1,
                           d ** -0.5, ws, ws.numel())
    torch.cuda.synchronize()
    k, v = torch.cat([ref().values(c.rows[0][:, :, : int(c.p[0])]), c.rows[0][:, :, int(c.p[0]) :].double()], 2)[:, 0]
    want = torch.softmax(q[:, 0].double() @ k.T * d ** -0.5, -1) @ v
    off = ((out[:, 0].double() - want).norm(dim=-1) / want.norm(dim=-1)).max().item()
    assert off <= 2.0 ** -8 + 2.0 ** -9, off
    c.close()


def test_packed_blocks_are_copied_whole_and_moved():
    x = normal(7, 2, 2, 16, 128, seed=1).to(torch.bfloat16)
    b = Blocks(x)
    K.kv_pack_blocks(b.h, 0, 1, b.a, b.q)
    raw = [b.buf[int(i) * b.block // 32 :][: b.block * 9 // 32].clone() for i in b.q]
    before = b.buf.clone()
    K.kv_copy_blocks(b.h, 1, [b.q[0], b.q[1], b.q[2]], [b.q[5], b.q[6], b.q[3]], [16, 0, 16])
    torch.cuda.synchronize()
    for i, want in ((5, 0), (6, 6), (3, 2), (4, 4)):
        assert torch.equal(b.buf[int(b.q[i]) * b.block // 32 :][: b.block * 9 // 32], raw[want])
    for i in (5, 3):
        at = int(b.q[i]) * b.block // 32
        before[at : at + b.block * 9 // 32] = b.buf[at : at + b.block * 9 // 32]
    assert torch.equal(before, b.buf)  # not a byte beside them
    b.close()


@pytest.mark.parametrize("d", [64, 128])
def test_tables_of_packed_blocks_compacted_and_forked(d):
    """Live packed blocks move together: the same attention afterwards, from fewer
    superpages; forks read the same blocks."""
    Hkv, Hq, bs, S = 2, 4, 16, 4
    block = 2 * Hkv * bs * d * 2
    buf = torch.zeros(64 * block, dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    h = K.kv_pool_create(buf, buf.numel(), bs, [(Hkv, d), (Hkv, d | K.KV_Q4)], err, page_bytes=block // 32, shuffle_seed=5)
    t, q4 = K.SeqTab(h, 0, S, 12), K.SeqTab(h, 1, S, 12)
    n = [150, 97, 33, 0]
    for s in range(S - 1):
        t.reserve(s, n[s])
        t.set_len(s, n[s])
    page = block // 32
    for s in range(S - 1):
        for j, i in enumerate(t.host()[0][s, : -(-n[s] // bs)]):
            buf[int(i) * page :][:block].view(torch.bfloat16)[:] = normal(block // 2, seed=100 * s + j).to(torch.bfloat16)
    # three a superpage: slot 0's first lies with two of slot 1's, its last two with room for one
    assert t.pack(q4, [2, 3], 1) == 2 and t.pack(q4, [1, 0], 1) == 15
    t.release(2)
    q4.release(2)
    t.release(1)
    q4.release(1)
    q4.fork(0, [3])
    t.fork(0, [3])
    table, lens = torch.empty(S, 12, dtype=torch.int32, device="cuda"), torch.empty(S, dtype=torch.int32, device="cuda")
    table4, lens4 = table.clone(), lens.clone()
    ws = torch.empty(K.kv_q4_workspace_bytes(h, 1, S, Hq, 12), dtype=torch.uint8, device="cuda")
    q = normal(S, Hq, d, seed=9).to(torch.bfloat16)
    q[3] = q[0]

    def attend():
        out = torch.empty(S, Hq, d, dtype=torch.bfloat16, device="cuda")
        t.sync(table, lens)
        q4.sync(table4, lens4)
        K.paged_decode_attn_q4(h, 0, 1, q, None, None, out, table, lens, 12, table4, lens4, 12, S, Hq, 0.1, ws, ws.numel())
        torch.cuda.synchronize()
        return out

    a = attend()
    # (another split over the warps: both off by 2^-8 of the value and 2^-11 of sum(p s c),
    # which is below a span, 8 here)
    assert ((a[0].float() - a[3].float()).abs() <= 2.0 ** -7 * a[0].float().abs() + 2.0 ** -7).all()
    assert (a[1:3] == 0).all() and torch.isfinite(a).all() and (a[0] != 0).any()
    ids = q4.host()[0].copy()
    assert K.kv_pool_compact(h) > 0
    assert (q4.host()[0] != ids).any()
    free = K.kv_pool_stats(h)["pages_unassigned"]
    K.kv_pool_trim(h)
    assert K.kv_pool_stats(h)["pages_unassigned"] > free
    assert torch.equal(attend(), a)
    assert K.kv_pool_get_error(h, None) == 0
    t.close()
    q4.close()
    K.kv_pool_destroy(h)
