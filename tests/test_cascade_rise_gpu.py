"""Shared-prefix attention where scores rise from key tile to key tile, in some
rows of a warp and not in others: the running maximum moves, and the
accumulator in tensor memory is rescaled by whole warps."""
import numpy as np
import pytest

import oracle
from tests.test_cascade_gpu import build, check, run

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G,Hkv,d", [(4, 2, 128), (1, 2, 128), (8, 1, 64), (5, 2, 64)])
def test_scores_that_rise_by_tile(G, Hkv, d):
    groups = [(list(range(40)), 1024)]
    pre = [1024 + 7 * i for i in range(40)]
    b = build(4400 + G + d, pre, groups, G, Hkv, d, 16)
    pages = b.pool.view(np.uint16).reshape(b.n_pages, 2, Hkv, 16, d)
    for j in range(64):  # K of 128-token tile t times 2^t, up to 2^4
        k = pages[b.table[0, j], 0]
        k[(k & 0x7FFF) != 0] += np.uint16(min(j // 8, 4) << 7)
    pool, db = run(b, groups, fused=False, lens=b.ctx_lens)
    check(db.out_f64(), oracle.batch_attention(b, pool=b.pool), "rising scores")
    assert pool.error() == 0
