"""The bf16 attention in pools with a 4-bit layout, down to pages of one bf16 row."""
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hkv,d,bs", [(1, 64, 16), (3, 64, 16), (1, 128, 16), (3, 128, 48), (5, 64, 48)])
def test_bf16_attention_beside_packed_blocks(Hkv, d, bs):
    """Contexts in bf16 alone, read by the 4-bit call (by bytes) and by the bf16
    ones (by rows)."""
    from tests import q4_ref

    Hq, n = 2 * Hkv, [70, 1, 300, 0, 48]
    c = q4_ref.PagedQ4(n, [0] * 5, Hq, Hkv, d, bs, 11, append=False)
    assert c.block // 32 % (2 * d) == 0
    q, scale = c.normal(5, Hq, d), d ** -0.5
    want, tol = c.reference(q, scale)
    out = torch.empty_like(q)
    ws = torch.empty(max(256, K.kv_workspace_bytes(c.h, 0, 5, Hq, c.max_blocks)), dtype=torch.uint8, device="cuda")
    q4_ref.check(c.run(q, scale), want, tol)
    K.paged_decode_attn(c.h, 0, q, out, c.table, c.lens, c.max_blocks, 5, Hq, scale, 0, ws, ws.numel())
    q4_ref.check(out, want, tol)
    out.fill_(float("nan"))
    K.paged_decode_attn_window(c.h, 0, q, None, None, out, c.table, c.lens, c.max_blocks, 5, Hq, scale, 0, 0, 0, ws, ws.numel())
    q4_ref.check(out, want, tol)
    # a prompt of each context's last token (the empty one has none)
    live = torch.tensor([0, 1, 2, 4], device="cuda")
    starts = torch.tensor([0, 1, 2, 3, 3, 4], dtype=torch.int32, device="cuda")
    nb = K.kv_prompt_workspace_bytes(c.h, 0, 5, Hq, 4, 1, c.max_blocks, 0, 0)
    ws = torch.empty(max(256, nb), dtype=torch.uint8, device="cuda")
    out = torch.empty(4, Hq, d, dtype=torch.bfloat16, device="cuda")
    K.paged_prompt_attn(c.h, 0, q[live].contiguous(), out, starts, 4, 1, c.table, c.lens, c.max_blocks, 5, Hq, scale, 0, 0, ws,
                        ws.numel())
    # (its weights are rounded to bf16, as the tolerance says)
    q4_ref.check(out, want[live], tol[live])
    assert c.error() == 0
    c.close()
