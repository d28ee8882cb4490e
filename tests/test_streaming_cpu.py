"""The windowed layer's handling of its arguments, on host tensors: the calls
that would launch something are recorded in place of being made."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

S, HQ, HKV, D, BS = 3, 4, 2, 64, 16


class HostPool:
    def __init__(self, n_pages=64):
        self.device = torch.device("cpu")
        self.handle = K.kv_pool_create(1 << 40, n_pages * 2 * HKV * BS * D * 2, BS, [(HKV, D)], (1 << 40) + (1 << 30))


@pytest.fixture
def layer(monkeypatch):
    from paper_2606_12950_gb300.streaming import WindowedLayer

    calls = []
    for name in ("kv_append_rotary", "paged_prompt_attn", "paged_decode_attn_window"):
        monkeypatch.setattr(K, name, lambda *a, name=name, **kw: calls.append((name, a)))
    monkeypatch.setattr(K, "kv_workspace_bytes", lambda *a: 256)
    monkeypatch.setattr(K, "kv_prompt_workspace_bytes", lambda *a: 0)
    monkeypatch.setattr(K.SeqTab, "sync", lambda *a: calls.append(("sync", a)))
    pool = HostPool()
    x = WindowedLayer(0, HQ, HKV, D, BS, S, 200, 40, 4, K.kv_rotary_freqs(D), pool=pool)
    x.calls = calls
    yield x
    x.tab.close()
    K.kv_pool_destroy(pool.handle)


def rows(n, heads, extra=0, dtype=torch.bfloat16):
    return torch.zeros((n, heads * D + extra), dtype=dtype)


def good(n):
    return {"q": rows(n, HQ), "k": rows(n, HKV), "v": rows(n, HKV)}


BAD = {
    "short": lambda n, h: rows(n - 1, h),
    "long": lambda n, h: rows(n + 1, h),
    "narrow": lambda n, h: rows(n, h)[:, 16:],
    "fp32": lambda n, h: rows(n, h, dtype=torch.float32),
    "fp16": lambda n, h: rows(n, h, dtype=torch.float16),
    "another device": lambda n, h: torch.empty((n, h * D), dtype=torch.bfloat16, device="meta"),
    "columns apart": lambda n, h: torch.zeros((n, 2 * h * D), dtype=torch.bfloat16)[:, ::2],
    "transposed": lambda n, h: torch.zeros((h * D, n), dtype=torch.bfloat16).t(),
    "heads apart": lambda n, h: torch.zeros((n, h, 2 * D), dtype=torch.bfloat16)[:, :, :D],
    "one row for all": lambda n, h: rows(1, h).expand(n, h * D),
    "flat": lambda n, h: torch.zeros(n * h * D, dtype=torch.bfloat16),
    "address": lambda n, h: rows(n, h, extra=8)[:, 1 : 1 + h * D],
    "row stride": lambda n, h: rows(n, h, extra=4)[:, : h * D],
}


@pytest.mark.parametrize("which", ["q", "k", "v"])
@pytest.mark.parametrize("how", sorted(BAD))
def test_rows_that_do_not_fit_are_refused_before_anything_changes(layer, which, how):
    layer.prompt([5, 0, 2], **good(7))
    layer.calls.clear()

    def state():
        tab, lens = layer.tab.host()
        return tab.copy(), lens.copy(), layer.pages_used()

    before = state()
    heads = HQ if which == "q" else HKV
    with pytest.raises(ValueError):
        layer.step(**{**good(S), which: BAD[how](S, heads)})
    with pytest.raises(ValueError):
        layer.prompt([20, 3, 0], **{**good(23), which: BAD[how](23, heads)})
    assert not layer.calls
    assert all(np.array_equal(a, b) for a, b in zip(before, state()))


def test_rows_as_they_come_are_taken(layer):
    """Column ranges of one projection, rows by head, wider rows, and no rows."""
    x = rows(7, HQ + 2 * HKV)
    q, k, v = x[:, : HQ * D], x[:, HQ * D : (HQ + HKV) * D], x[:, (HQ + HKV) * D :]
    layer.prompt([5, 0, 2], q, k, v)
    name, a = layer.calls[1]
    assert name == "kv_append_rotary" and (a[3] is q and a[6] is k and a[8] is v)
    assert a[4] == a[7] == a[9] == (HQ + 2 * HKV) * D and a[12] == 7
    layer.step(torch.zeros((S, HQ, D), dtype=torch.bfloat16), torch.zeros((S, HKV, D), dtype=torch.bfloat16), rows(S, HQ))
    layer.calls.clear()
    assert layer.prompt([0, 0, 0], *(y[:0] for y in (q, k, v))).shape == (0, HQ, D)
    assert not layer.calls
    assert layer.tab.lens().tolist() == [6, 0, 3]
