"""Pools of bf16 and 4-bit blocks whose pages are no whole number of bf16 rows:
the bf16 attention, which finds a block by its row, refuses such a layout."""
import pytest

from paper_2606_12950_gb300 import kvpool as K

BASE, ERR, X = 1 << 40, (1 << 40) + (1 << 30), 1 << 41
Q = K.KV_Q4


def code(call, *args):
    with pytest.raises(K.KVError) as e:
        call(*args)
    return e.value.code


def attention_calls(h, layout, Hq):
    """The bf16 attention calls of the library on one layout (on addresses that are
    no memory: only where they are refused)."""
    batch = dict(layout=layout, S=1, Hq=Hq, max_blocks=4, scale=0.1, q=X, out=X, dev_table=X, dev_ctx_lens=X, workspace=X,
                 ws_bytes=1 << 30)
    return {
        "workspace": lambda: K.kv_workspace_bytes(h, layout, 1, Hq, 4),
        "decode": lambda: K.paged_decode_attn(h, layout, X, X, X, X, 4, 1, Hq, 0.1, 0, X, 1 << 30),
        "append": lambda: K.paged_decode_attn_append(h, layout, X, X, X, X, X, X, 4, 1, Hq, 0.1, 0, X, 1 << 30),
        "window": lambda: K.paged_decode_attn_window(h, layout, X, None, None, X, X, X, 4, 1, Hq, 0.1, 8, 0, 0, X, 1 << 30),
        "prompt workspace": lambda: K.kv_prompt_workspace_bytes(h, layout, 1, Hq, 1, 1, 4, 0, 0),
        "prompt": lambda: K.paged_prompt_attn(h, layout, X, X, X, 1, 1, X, X, 4, 1, Hq, 0.1, 0, 0, X, 1 << 30),
        "cascade workspace": lambda: K.kv_cascade_workspace_bytes(h, layout, 1, Hq, 4),
        "several batches": lambda: K.paged_decode_attn_multi(h, [batch]),
        "no workspace": lambda: K.paged_decode_attn_noalloc(h, layout, X, X, X, X, 4, 1, Hq, 0.1),
    }


@pytest.mark.parametrize("layouts,bs,page,bad", [
    ([(1, 128), (1, 128 | Q)], 16, 128, [0]),                                # half a row
    ([(1, 64), (1, 64 | Q), (1, 128), (1, 128 | Q)], 16, 128, [2]),          # the only size for both
    ([(3, 128), (3, 128 | Q)], 16, 384, [0]),                                # a row and a half
    ([(1, 64), (1, 64 | Q), (1, 128)], 48, 384, [2]),
    ([(2, 128), (2, 128 | Q)], 16, 512, []),
    ([(1, 64), (1, 64 | Q)], 16, 128, []),
])
def test_pages_of_no_whole_rows(layouts, bs, page, bad):
    h = K.kv_pool_create(BASE, 64 * 2 * 4 * bs * 128 * 2, bs, layouts, ERR, page_bytes=page)
    for layout, (Hkv, d) in enumerate(layouts):
        if d & Q:
            continue
        if layout in bad:
            for name, call in attention_calls(h, layout, Hkv).items():
                assert code(call) == K.KV_ERR_UNSUPPORTED, name
        else:
            try:
                assert K.kv_workspace_bytes(h, layout, 1, Hkv, 4) > 0
            except K.KVError as e:
                assert e.code == K.KV_ERR_CUDA  # (no GPU)
        # what goes by bytes serves every layout
        ids = K.kv_alloc_blocks(h, layout, 2)
        K.kv_free_blocks(h, layout, ids)
    K.kv_pool_destroy(h)
