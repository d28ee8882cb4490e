"""4-bit decode attention over blocks that are packed in part, and runs merged by
parts for every group of query heads."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


def packed_further(c, tiles):
    """Moves tiles[s] tiles of 16 tokens of the block after sequence s's packed ones
    into 4 bits as well: the block is packed as it stands (rows past the context are
    no numbers), the packed length ends inside it, and its bf16 form serves the rest."""
    K.kv_pool_trim(c.h)
    for s, k in enumerate(tiles):
        b = int(c.p[s]) // c.bs
        assert 0 <= 16 * k < c.bs and c.p[s] + 16 * k <= c.n[s]
        if k:
            new = K.kv_alloc_blocks(c.h, 1, 1)
            K.kv_pack_blocks(c.h, 0, 1, [c.host_table[s, b]], new)
            c.table4[s, b] = int(new[0])
            c.p[s] += 16 * k
    c.packed = torch.from_numpy(c.p.astype(np.int32)).cuda()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bs", [32, 48, 64, 256])
@pytest.mark.parametrize("append", [True, False])
def test_packed_lengths_inside_a_block(bs, d, append):
    from tests import q4_ref

    t = bs // 16
    n = [3 * bs + 17, 2 * bs - 1, bs, 5 * bs + 16 * (t - 1) + 1, 900, 16 + append, 4 * bs + 20]
    p = [3 * bs, bs, 0, 5 * bs, 900 // bs * bs, 0, 0]
    k = [1, t - 1 if bs > 32 else 0, t - 1, t - 1, (900 % bs - append) // 16, 1, t - 1]
    c = q4_ref.PagedQ4(n, p, 8, 2, d, bs, 5, append=append)
    packed_further(c, k)
    q = c.normal(c.S, 8, d)
    out = c.run(q, d ** -0.5)
    torch.cuda.synchronize()
    q4_ref.check(out, *c.reference(q, d ** -0.5))
    assert c.error() == 0
    c.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(16, 4), (20, 4), (32, 4), (4, 4)])
@pytest.mark.parametrize("kind", ["two", "among short ones"])
def test_merge_by_parts(kind, Hq, Hkv, d):
    """Eight runs a CTA and more, most of them empty or short: partial states are
    merged by the CTA that a run starts in, whatever the group."""
    from tests import q4_ref

    n, p = np.zeros(320, np.int64), np.zeros(320, np.int64)
    if kind == "two":
        n[100], p[100], n[319], p[319] = 20007, 19984, 5, 0
    else:
        n[:] = np.arange(320) % 45
        p[:] = (n - 1).clip(0) // 16 * 16
        n[160], p[160] = 30011, 29984
    c = q4_ref.PagedQ4(n, p, Hq, Hkv, d, 16, 5)
    q = c.normal(c.S, Hq, d)
    out = c.run(q, d ** -0.5)
    torch.cuda.synchronize()
    q4_ref.check(out, *c.reference(q, d ** -0.5))
    assert (out[torch.from_numpy(n == 0).cuda()] == 0).all() and c.error() == 0
    assert torch.equal(c.run(q, d ** -0.5), out)
    c.close()
