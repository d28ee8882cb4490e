"""The windowed decode call runs the tensor-core kernel whatever the pool's
variant is and however wide the window: its bits do not depend on either."""
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 8, 2), (64, 10, 2), (128, 8, 1)])
@pytest.mark.parametrize("append", [False, True])
def test_cuda_core_variant_leaves_every_window_alone(d, Hq, Hkv, append):
    from tests.paged_ref import Paged, check

    n = [700, 16, 333, 1]
    c = Paged(n, [1] * 4, Hq, Hkv, d, 16, seed=d + Hq)
    q = c.normal(4, Hq, d)
    k, v = (c.normal(4, Hkv, d), c.normal(4, Hkv, d)) if append else (None, None)
    reach = c.max_blocks * 16

    def attend(window, splits, nb=None):
        out = torch.full((4, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        nb = nb or K.kv_workspace_bytes(c.h, 0, 4, Hq, c.max_blocks, splits)
        ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda")
        K.paged_decode_attn_window(c.h, 0, q, k, v, out, c.table, c.lens, c.max_blocks, 4, Hq, d ** -0.5, window, 3,
                                   splits, ws, nb)
        torch.cuda.synchronize()
        assert c.error() == 0
        return out

    for window in (0, reach, 10 ** 9, 100):
        for splits in (5, 60):
            K.kv_set_attn_variant(c.h, 0)
            nb = K.kv_workspace_bytes(c.h, 0, 4, Hq, c.max_blocks, splits)
            want = attend(window, splits)
            K.kv_set_attn_variant(c.h, 1)
            assert torch.equal(attend(window, splits, nb), want), (window, splits)
        # the pool's variant sizes the workspace of its default split (the
        # CUDA-core kernel has none for 8 heads a group: sized before)
        K.kv_set_attn_variant(c.h, 0)
        nb = K.kv_workspace_bytes(c.h, 0, 4, Hq, c.max_blocks, 0) if Hq // Hkv == 8 else None
        K.kv_set_attn_variant(c.h, 1)
        out = attend(window, 0, nb)
        check(out, *c.reference(q, d ** -0.5, window if window < reach else 0, 3))
    c.close()
