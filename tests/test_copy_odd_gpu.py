"""Page copies of layouts whose blocks and rows are no powers of two: whole
blocks, and the first rows of each head's K and V."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402
from paper_2606_12950_gb300.runner import DevicePool  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 81, 400])
@pytest.mark.parametrize("Hkv,d,bs", [(8, 16, 7), (4, 40, 8), (16, 24, 5)])
@pytest.mark.parametrize("partial", [False, True])
def test_copies_of_odd_blocks(n, Hkv, d, bs, partial):
    page = 2 * Hkv * bs * d * 2
    assert page % 256 == 0
    p = DevicePool(2 * n + 5, page, bs, [(Hkv, d)])
    rows = p.buf.view(torch.int16).view(-1, 2, Hkv, bs, d)
    rows.copy_(torch.randint(-2 ** 15, 2 ** 15, rows.shape, dtype=torch.int16, device="cuda"))
    rng = np.random.default_rng(n)
    ids = rng.permutation(K.kv_alloc_blocks(p.handle, 0, 2 * n + 5))
    src, dst = ids[:n], ids[n : 2 * n]
    tokens = rng.integers(0, bs + 1, n) if partial else None
    want = rows.clone()
    for i in range(n):
        m = int(tokens[i]) if partial else bs
        want[dst[i], :, :, :m] = want[src[i], :, :, :m]
    K.kv_copy_blocks(p.handle, 0, src, dst, tokens)
    torch.cuda.synchronize()
    assert torch.equal(rows, want)
    p.close()
