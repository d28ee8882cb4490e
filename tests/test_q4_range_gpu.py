"""4-bit decode attention over V rows whose scales and least values lie far apart:
each group of 64 columns is as exact as its own numbers allow."""
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu

N, P, SCALE = [700, 333, 40, 1000], [688, 320, 32, 0], 128 ** -0.5
SPECIAL = 100  # a token in 4 bits of the first two sequences


def generator(s, kv):
    g = torch.Generator(device="cuda")
    g.manual_seed(10 * s + kv + 1)
    return g


def queries(d, Hq=8):
    return torch.randn(len(N), Hq, d, device="cuda", generator=generator(9, 0)).to(torch.bfloat16)


def cache(d, change, append, q, dismissed=False):
    """Hkv = 2; change(x, s) edits the V rows [2, n, d] of sequence s in fp32.
    dismissed: token SPECIAL's keys turn away from every query of their KV head, so
    that its weight is below 2^-60 of the largest."""
    from tests import q4_ref

    def make(kv, s, m):
        x = torch.randn(2, m, d, device="cuda", generator=generator(s, kv))
        if kv == 1:
            change(x, s)
        elif dismissed and m > SPECIAL:
            heads = q[s].float().view(2, -1, d)
            x[:, SPECIAL] = -12.0 * heads.sum(1)
        return x.to(torch.bfloat16)

    return q4_ref.PagedQ4(N, P, q.shape[1], 2, d, 16, 4, append=append, make=make)


def grain(c, q):
    """What weights that are small beside the largest lose: fp16 holds the largest
    weight * scale of a head and a group at 2^7 or more, so one below its normal
    numbers is off by 2^-25, 2^-32 of the largest, and codes are 15 at most."""
    from tests.q4_ref import quantised, values

    G, t = c.Hq // c.Hkv, torch.zeros(c.S, c.Hkv, c.Hq // c.Hkv, c.d, dtype=torch.float64, device="cuda")
    for s in range(c.S):
        n, p = int(c.n[s]), int(c.p[s])
        if p == 0:
            continue
        x = c.rows[s]
        k = torch.cat([values(x[0, :, :p]), x[0, :, p:].double()], 1)
        sc = quantised(x[1, :, :p])[1].double().squeeze(-1).nan_to_num(0.0)  # [Hkv, p, groups]
        w = torch.softmax(q[s].view(c.Hkv, G, c.d).double() @ k.transpose(1, 2) * SCALE, -1)[..., :p]
        most = (w.unsqueeze(-1) * sc.unsqueeze(1)).amax(2)  # [Hkv, G, groups]
        t[s] = (15 * n * 2.0 ** -32 * most).repeat_interleave(64, -1)
    return t.view(c.S, c.Hq, c.d)


def check(c, q, nan=None):
    """Against 64 bits; nan [S, Hq, d]: outputs that are NaN and nothing else."""
    from tests import q4_ref

    out = c.run(q, SCALE)
    torch.cuda.synchronize()
    want, tol = c.reference(q, SCALE)
    tol = tol + grain(c, q)
    if nan is not None:
        # (64-bit weights times NaN leave no finite column of a row: those of the
        # groups without one are computed by themselves)
        assert torch.equal(torch.isnan(out), nan)
        want, tol, out = want.masked_fill(nan, 0.0), tol.masked_fill(nan, 0.0), out.masked_fill(nan, 0.0)
    q4_ref.check(out, want, tol)
    assert c.error() == 0
    c.close()


@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("e", [20, 24, 30, 40, 60, -24, -40])
def test_groups_of_other_scales(e, append):
    """Columns 64 to 127 are 2^e times the others'."""
    def change(x, s):
        x[..., 64:] *= 2.0 ** e

    q = queries(128)
    check(cache(128, change, append, q), q)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("e", [16, 24, 30, 50, 70])
def test_a_large_token_of_no_weight(e, d):
    """One token's V row is 2^e times the others', its weight nothing: neither its
    own group nor the other loses a digit."""
    def change(x, s):
        if x.shape[1] > SPECIAL:
            x[:, SPECIAL, d - 64 :] *= 2.0 ** e

    q = queries(d)
    check(cache(d, change, True, q, dismissed=True), q)


@pytest.mark.parametrize("e", [16, 30, 50])
def test_a_large_token_with_weight(e):
    """The same with a weight like the others'."""
    def change(x, s):
        if x.shape[1] > SPECIAL:
            x[0, SPECIAL, :64] *= 2.0 ** e
            x[1, SPECIAL + 40 :, 64:] *= 2.0 ** -e  # (and all that come after are small)

    q = queries(128)
    check(cache(128, change, True, q), q)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 2.0 ** 100])
@pytest.mark.parametrize("dismissed", [True, False])
def test_a_group_without_numbers(bad, dismissed):
    """Columns 64 to 127 of one token hold no number: the others stay exact.
    (2^100: a span over 2^80 makes the group NaN.)"""
    def change(x, s):
        if s == 0:
            x[1, SPECIAL, 70] = bad

    q = queries(128)
    c = cache(128, change, True, q, dismissed)
    nan = torch.zeros(len(N), 8, 128, dtype=torch.bool, device="cuda")
    nan[0, 4:, 64:] = True
    check(c, q, nan)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", [2.0 ** 72, 2.0 ** 80, -(2.0 ** 100), 2.0 ** 122])
@pytest.mark.parametrize("which", ["all", "one group", "alternating"])
def test_constant_groups_of_large_values(value, which, d):
    """Groups of one value have scale 0; the sums of weight * value stay in range."""
    def change(x, s):
        if which == "all":
            x[:] = value
        elif which == "one group":
            x[..., :64] = value
        else:
            x[:] = value
            x[:, ::2] = -value

    q = queries(d)
    check(cache(d, change, True, q), q)


@pytest.mark.parametrize("e", [-30, -60, -70])
def test_small_scales(e):
    """V rows of 2^e, with a constant group beside them or not."""
    def change(x, s):
        x *= 2.0 ** e
        if s == 1:
            x[..., :64] = 1.0

    q = queries(128)
    check(cache(128, change, False, q), q)


@pytest.mark.parametrize("d", [64, 128])
def test_scales_that_change_along_a_run(d):
    """Scales rise and fall by up to 2^100 from stretch to stretch of a context, and
    so do the scores, so that what was largest once is not later.  (As many contexts
    as warps, over the same blocks, so that a warp takes one from end to end.)"""
    from tests import q4_ref

    n, S = 3000, 2560
    g = generator(3, 3)
    q = torch.randn(1, 1, d, device="cuda", generator=g).to(torch.bfloat16)

    def make(kv, s, m):
        x = torch.randn(1, m, d, device="cuda", generator=g)
        step = torch.arange(m, device="cuda") // 250
        if kv == 0:  # scores of about 0, 12, -3, 30, ..
            up = torch.tensor([0.0, 12, -3, 30, 29, 2, 45, 44, 0, 40, 46, 45], device="cuda")[step]
            x = x + up[None, :, None] * q[0].float() / (q.float().square().sum() * SCALE)
        else:
            x = x * torch.exp2(torch.tensor([0.0, 30, -30, -10, 40, 10, -20, 25, 60, 5, -15, 0], device="cuda")[step])[None, :, None]
        return x.to(torch.bfloat16)

    c = q4_ref.PagedQ4([n], [n // 16 * 16 - 16], 1, 1, d, 16, 4, append=False, make=make)
    table, table4 = c.table.expand(S, -1).contiguous(), c.table4.expand(S, -1).contiguous()
    lens, packed = c.lens.expand(S).contiguous(), c.packed.expand(S).contiguous()
    out = torch.empty(S, 1, d, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(K.kv_q4_workspace_bytes(c.h, 1, S, 1, c.max_blocks), dtype=torch.uint8, device="cuda")
    K.paged_decode_attn_q4(c.h, 0, 1, q.expand(S, 1, d).contiguous(), None, None, out, table, lens, c.max_blocks, table4, packed,
                           c.max_blocks4, S, 1, SCALE, ws, ws.numel())
    torch.cuda.synchronize()
    want, tol = c.reference(q, SCALE)
    q4_ref.check(out, want.expand(S, 1, d), (tol + grain(c, q)).expand(S, 1, d))
    c.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", [2.0 ** 123, -(2.0 ** 124), 2.0 ** 126, 3.0e38])
@pytest.mark.parametrize("column", [6, 7, 63])
def test_large_values_in_bf16_rows(column, value, d):
    """One bf16 row holds a value near fp32's last, in an even or odd column: the
    output is finite and right, in contexts with tokens in 4 bits and without."""
    from tests import q4_ref

    def change(x, s):
        m = x.shape[1]
        for t in (m - 1, m - 5, SPECIAL):
            if P[s] <= t < m:
                x[:, t, column] = value * 2.0 ** (-3 * (t != SPECIAL))

    q = queries(d)
    c = cache(d, change, True, q)
    out = c.run(q, SCALE)
    torch.cuda.synchronize()
    want, tol = c.reference(q, SCALE)
    assert torch.isfinite(out).all()
    q4_ref.check(out, want, tol + grain(c, q))
    assert c.error() == 0
    c.close()


@pytest.mark.parametrize("d", [64, 128])
def test_a_token_with_all_the_weight_gives_its_row(d):
    """The largest weight loses nothing where weights are rounded: a context of one
    token gives its V row bit for bit, one whose other tokens weigh under 2^-40 the
    row of the token that is left, rounded once (2^-8 of the value).  Besides, s c is
    weighed with the rounded weight and z with the fp32 one, whose exponent, a
    difference of numbers in [64, 128) with a spacing of 2^-17, is off by 2^-18: the
    weight by ln 2 of that, z by as much of V's largest, and the fp32 sums by 2^-20 of it:
    under 2^-17 together."""
    from tests import q4_ref

    S, at = 40, 37  # the token: in 4 bits in half of the sequences, the others in bf16
    g = generator(5, 5)
    q = torch.randn(2 * S, 8, d, device="cuda", generator=g).to(torch.bfloat16)
    q[:, 1:4], q[:, 5:] = q[:, :1], q[:, 4:5]  # (a KV head's queries alike)

    def make(kv, s, m):
        x = torch.randn(2, m, d, device="cuda", generator=g)
        if kv == 0 and m > at:
            h = q[s, ::4].float()
            x[:, at] = h * ((55 + 0.3 * s) * d ** 0.5 / h.square().sum(-1, keepdim=True))
        return x.to(torch.bfloat16)

    c = q4_ref.PagedQ4([1] * S + [60] * S, [0] * S + [48 * (s % 2) for s in range(S)], 8, 2, d, 16, 4, append=False, make=make)
    out = c.run(q, d ** -0.5)
    torch.cuda.synchronize()
    for s in range(2 * S):
        x = c.rows[s][1]
        if s < S:
            assert torch.equal(out[s].view(2, 4, d), x[:, :1].expand(2, 4, d))
            continue
        row = (q4_ref.values(x) if c.p[s] else x.double())[:, at : at + 1]
        assert ((out[s].view(2, 4, d).double() - row).abs() <= 2.0 ** -8 * row.abs() + 2.0 ** -17 * x.double().abs().max()).all()
    assert c.error() == 0
    c.close()
