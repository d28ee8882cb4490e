"""Prompt chunks longer than the call's max_q: the items are as many as max_q
asks for, so rows may have none, and the error word says so."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


def attend(c, q, max_q):
    out = torch.zeros((c.T, c.Hq, c.d), dtype=torch.bfloat16, device="cuda")
    nb = K.kv_prompt_workspace_bytes(c.h, 0, c.S, c.Hq, c.T, max_q, c.max_blocks, 0, 0)
    # zeros: rows without records then merge to nothing
    ws = torch.zeros(max(nb, 256), dtype=torch.uint8, device="cuda")
    K.paged_prompt_attn(c.h, 0, q, out, c.starts, c.T, max_q, c.table, c.lens, c.max_blocks, c.S, c.Hq, c.d ** -0.5,
                        0, 0, ws, nb)
    torch.cuda.synchronize()
    return out


# one sequence; the long chunk first, in the middle, last; more sequences than
# are put in order (32), and enough for a second item a CTA
@pytest.mark.parametrize("nq,max_q", [([300], 40), ([300, 5, 5], 5), ([5, 300, 5], 5), ([5, 5, 300], 5), ([129], 128),
                                      ([300] + [2] * 50, 2), ([2] * 50 + [300], 2), ([90] * 160 + [200], 90)])
@pytest.mark.parametrize("d", [64, 128])
def test_a_chunk_longer_than_the_bound_is_reported(nq, max_q, d):
    from tests.paged_ref import Paged, check

    nq = np.array(nq)
    c = Paged(nq + 20, nq, 4, 1, d, 16, 3)
    q = c.normal(c.T, 4, d)
    attend(c, q, max_q)
    assert c.error() == K.KV_ERR_DEVICE_BOUNDS
    check(attend(c, q, int(nq.max())), *c.reference(q, d ** -0.5, 0, 0))
    assert c.error() == 0
    c.close()
