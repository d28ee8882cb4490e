"""The prompt kernel where a CTA takes several items: of two Q tiles, over masked
and unmasked tiles, in order of their key ranges (32 sequences at most) or of the
sequences; and bad values in V beside key splits and at d = 64."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


def attend(c, q, window, sinks):
    out = torch.full((c.T, c.Hq, c.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    max_q = int(c.nq.max())
    nb = K.kv_prompt_workspace_bytes(c.h, 0, c.S, c.Hq, c.T, max_q, c.max_blocks, window, sinks)
    ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda") if nb else None
    K.paged_prompt_attn(c.h, 0, q, out, c.starts, c.T, max_q, c.table, c.lens, c.max_blocks, c.S, c.Hq, c.d ** -0.5,
                        window, sinks, ws, nb)
    torch.cuda.synchronize()
    return out, nb


def items(c):
    """Items of the call: two Q tiles of floor(128 / G) tokens each, per KV head."""
    TT = 2 * (128 // (c.Hq // c.Hkv))
    return sum(-(-int(x) // TT) for x in c.nq) * c.Hkv


def reference(c, q, window, sinks):
    """The definition in 64 bits on the GPU, a sequence and head at a time, and
    sum of weight * |v| (finite values).  (Paged.reference is the host's, slow at
    these sizes, and its second sum leaves out every head of a token that has a bad
    value in one, weights that are rounded all the same.)  A bad value counts where
    its token is seen."""
    out = torch.zeros(c.T, c.Hq, c.d, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    G, at = c.Hq // c.Hkv, 0
    for s in range(c.S):
        nq, n = int(c.nq[s]), int(c.n[s])
        if nq == 0:
            continue
        p, j = torch.arange(n - nq, n, device="cuda").view(-1, 1), torch.arange(n, device="cuda")
        seen = j <= p
        if window:
            seen &= (j > p - window) | (j < sinks)
        some = seen.any(0)  # given-up blocks stay out
        j, seen = j[some], seen[:, some]
        blk = torch.from_numpy(c.host_table[s].astype(np.int64)).cuda()[j // c.bs]
        k, v = c.pool[blk, :, :, j % c.bs].double().permute(1, 2, 0, 3)
        for h in range(c.Hq):
            x = (q[at : at + nq, h].double() @ k[h // G].T * c.d ** -0.5).masked_fill(~seen, -np.inf)
            w = torch.softmax(x, -1)
            bad = ~torch.isfinite(v[h // G])
            fine = torch.where(bad, 0.0, v[h // G])
            o = w @ fine
            for t in bad.any(1).nonzero().flatten().tolist():
                o[:, bad[t]] += torch.where(seen[:, t : t + 1], w[:, t : t + 1] * v[h // G, t, bad[t]], 0.0)
            out[at : at + nq, h], bound[at : at + nq, h] = o, w @ fine.abs()
        at += nq
    return out, bound


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,nq,window,sinks", [
    # one document, and causal prompts of unequal lengths: sorted, few masked tiles
    ([3001], [3001], 0, 0), ([2500, 700, 1700, 130, 1], [2500, 700, 1700, 130, 1], 0, 0),
    # behind contexts, windowed: head and gap tiles, evicted blocks
    ([5000, 900, 4100], [1500, 900, 1100], 700, 4), ([4000, 3000], [2100, 900], 150, 200),
    # 32 sequences are sorted, 33 are not
    (list(range(40, 40 + 32 * 23, 23)), list(range(40, 40 + 32 * 23, 23)), 0, 0),
    (list(range(40, 40 + 33 * 23, 23)), list(range(40, 40 + 33 * 23, 23)), 0, 0),
    (list(range(300, 300 + 70 * 9, 9)), list(range(70, 70 + 70 * 3, 3)), 190, 5),
])
def test_several_items_a_cta(d, n, nq, window, sinks):
    from tests.paged_ref import Paged, check, holds

    Hq, Hkv = 40, 8  # TQ 25: tokens of an item are no power of two, three rows of each Q tile idle
    c = Paged(n, nq, Hq, Hkv, d, 16, seed=len(n) + d, held=holds(n, nq, window, sinks, 16))
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert items(c) > 2 * sms  # some CTA takes a third item: rounds forwards and backwards
    q = c.normal(c.T, Hq, d)
    out, nb = attend(c, q, window, sinks)
    assert nb == 0 and c.error() == 0
    check(out, *reference(c, q, window, sinks))
    # an item's bits do not depend on which CTA takes it, or after which other
    assert torch.equal(attend(c, q, window, sinks)[0], out)
    c.close()


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 16, 16), (128, 16, 16), (64, 32, 4), (128, 32, 4)])
def test_several_items_a_cta_of_other_groups(d, Hq, Hkv):
    """Groups of 1 (items of 256 tokens) and 8 (of 32)."""
    from tests.paged_ref import Paged, check

    n = [2900, 1100, 900] if Hq == Hkv else [1200, 500, 900]
    c = Paged(n, n, Hq, Hkv, d, 16, seed=Hq + d)
    assert items(c) > 152
    q = c.normal(c.T, Hq, d)
    out, nb = attend(c, q, 0, 0)
    assert nb == 0 and c.error() == 0
    check(out, *reference(c, q, 0, 0))
    c.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_bad_values_with_several_items_a_cta(d, bad):
    """In V of tokens that some queries of an item see and others do not: at the
    diagonal and at the window's edge, of several items of one CTA."""
    from tests.paged_ref import Paged, check

    window, sinks = 120, 3
    n = nq = [900, 600, 500]
    c = Paged(n, nq, 40, 8, d, 16, seed=d, held=None)
    b = c.host_table
    for s, tok, g, col in ((0, 0, 0, 3), (0, 430, 2, slice(None)), (0, 899, 7, 5), (1, 431, 1, 0), (1, 432, 5, d - 1),
                           (2, 2, 3, 40), (2, 480, 6, slice(None))):
        c.pool[b[s, tok // 16], 1, g, tok % 16, col] = bad
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert items(c) > 2 * sms
    q = c.normal(c.T, 40, d)
    out, nb = attend(c, q, window, sinks)
    assert nb == 0 and c.error() == 0
    check(out, *reference(c, q, window, sinks))
    c.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (3000, 5)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_bad_values_with_key_splits(d, window, sinks, bad):
    """Noted rows in the first, a middle and the last split's tiles."""
    from tests.paged_ref import Paged, check, holds

    n, nq = [6007], [9]
    c = Paged(n, nq, 8, 2, d, 16, seed=5, held=holds(n, nq, window, sinks, 16))
    b = c.host_table[0]
    for tok, g, col in ((6006, 0, 9), (6001, 1, slice(None)), (4000, 0, 33), (6007 - 3000 - 1, 1, 7) if window else (7, 1, 7)):
        if b[tok // 16] >= 0:
            c.pool[b[tok // 16], 1, g, tok % 16, col] = bad
    q = c.normal(9, 8, d)
    out, nb = attend(c, q, window, sinks)
    assert nb > 0 and c.error() == 0
    check(out, *reference(c, q, window, sinks))
    c.close()


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_bad_values_at_head_dim_64(window, sinks, bad):
    from tests.paged_ref import Paged, check

    c = Paged([150], [150], 8, 2, 64, 16, seed=7)
    b = c.host_table[0]
    c.pool[b[50 // 16], 1, 1, 50 % 16, 9] = bad
    c.pool[b[149 // 16], 1, 0, 149 % 16] = bad
    q = c.normal(c.T, 8, 64)
    out, _ = attend(c, q, window, sinks)
    check(out, *reference(c, q, window, sinks))
    assert c.error() == 0
    c.close()


def test_another_stream_after_the_current_one():
    """Buffers filled on the current stream, waited for by the call's."""
    from tests.paged_ref import Paged

    c = Paged([900, 300], [700, 300], 8, 2, 128, 16, seed=5)
    q = c.normal(c.T, 8, 128)
    want, nb = attend(c, q, 0, 0)
    st = torch.cuda.Stream()
    out = torch.full_like(q, float("nan"))
    st.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(max(nb, 256), dtype=torch.uint8, device="cuda")
    K.paged_prompt_attn(c.h, 0, q, out, c.starts, c.T, 700, c.table, c.lens, c.max_blocks, 2, 8, 128 ** -0.5, 0, 0, ws,
                        nb, st)
    st.synchronize()
    assert torch.equal(out, want)
    c.close()
