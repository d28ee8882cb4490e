"""The windowed layer's handling of its arguments, on host tensors: the calls
that would launch something are recorded in place of being made, and streams are
objects that write down what waits for what."""
import contextlib

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

S, HQ, HKV, D, BS = 3, 4, 2, 64, 16


class HostPool:
    def __init__(self, n_pages=64):
        self.device = torch.device("cpu")
        self.handle = K.kv_pool_create(1 << 40, n_pages * 2 * HKV * BS * D * 2, BS, [(HKV, D)], (1 << 40) + (1 << 30))


class Streams:
    """torch.cuda's streams: the current one, and each one's waits in order."""

    class Stream:
        def __init__(self, handle, log):
            self.cuda_stream, self.log, self.stream_id = handle, log, handle + 1 if handle else 0

        def wait_stream(self, other):
            self.log.append(("wait", self.cuda_stream, other.cuda_stream))

        def wait_event(self, event):
            self.log.append(("wait", self.cuda_stream, event))

        def record_event(self):
            return f"event of {self.cuda_stream}"

    def __init__(self, monkeypatch):
        self.log = log = []
        self.current = [self.Stream(100, log)]

        class External(self.Stream):
            def __init__(self, handle, device=None):
                super().__init__(handle, log)
                self.stream_id = handle

        @contextlib.contextmanager
        def use(s):
            self.current.append(s)
            try:
                yield
            finally:
                self.current.pop()

        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.current[-1])
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: self.current[-1].cuda_stream, raising=False)
        monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: self.Stream(0, log))
        monkeypatch.setattr(torch.cuda, "ExternalStream", External)
        monkeypatch.setattr(torch.cuda, "stream", use)
        monkeypatch.setattr(torch.Tensor, "record_stream",
                            lambda x, s: log.append(("keep", x.data_ptr(), s.cuda_stream)))

    def new(self, handle):
        return self.Stream(handle, self.log)


@pytest.fixture
def streams(monkeypatch):
    return Streams(monkeypatch)


@pytest.fixture
def layer(monkeypatch, streams):
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


def launched_on(layer, streams, monkeypatch):
    """Makes every recorded call write (name, handle of its stream, handle of the
    stream that was current) into the streams' log, and every tensor the layer
    makes the stream that was current."""
    def note(name):
        def call(*a, **kw):
            s = kw.get("stream", a[-1] if a else None)
            streams.log.append((name, getattr(s, "cuda_stream", s), streams.current[-1].cuda_stream))
            return 0
        return call

    for name in ("kv_append_rotary", "paged_prompt_attn", "paged_decode_attn_window", "kv_pool_compact"):
        monkeypatch.setattr(K, name, note(name))
    for name in ("sync", "fork"):
        monkeypatch.setattr(K.SeqTab, name, note(name))
    empty = torch.empty

    def made(*a, **kw):
        streams.log.append(("made", streams.current[-1].cuda_stream))
        return empty(*a, **kw)

    monkeypatch.setattr(torch, "empty", made)


def kernels(log):
    return [e for e in log if e[0] not in ("wait", "keep", "made")]


def calls_of(layer, stream, **rows_):
    yield lambda: layer.prompt([5, 0, 2], **good(7), stream=stream)
    yield lambda: layer.step(**good(S), stream=stream)
    yield lambda: layer.fork(0, [1], stream=stream)
    yield lambda: layer.compact(stream=stream)


def test_the_current_stream_is_the_default(layer, streams, monkeypatch):
    launched_on(layer, streams, monkeypatch)
    for handle in (100, 7, 0):
        streams.current[0].cuda_stream = handle
        for call in calls_of(layer, None):
            streams.log.clear()
            call()
            assert kernels(streams.log) and all(e[1:] == (handle, handle) for e in kernels(streams.log))
            assert all(e == ("made", handle) for e in streams.log if e[0] == "made")


def test_on_another_stream(layer, streams, monkeypatch):
    """It waits for the current stream first, what the call allocates is its own,
    and the caller's rows and the layer's buffers are kept until it is done."""
    launched_on(layer, streams, monkeypatch)
    side = streams.new(55)
    for call in calls_of(layer, side):
        streams.log.clear()
        call()
        k = kernels(streams.log)
        assert k and all(e[1:] == (55, 55) for e in k)
        assert streams.log.index(("wait", 55, 100)) < streams.log.index(k[0])
        assert all(e == ("made", 55) for e in streams.log if e[0] == "made")
        assert streams.current[-1].cuda_stream == 100
    streams.log.clear()
    r = good(S)
    out = layer.step(**r, stream=side)
    for x in r.values():
        assert ("keep", x.data_ptr(), 55) in streams.log
    assert ("keep", out.data_ptr(), 100) in streams.log  # the caller may read it where it called


def test_a_call_waits_for_the_one_before_on_another_stream(layer, streams, monkeypatch):
    launched_on(layer, streams, monkeypatch)
    a, b = streams.new(55), streams.new(66)
    layer.prompt([5, 0, 2], **good(7), stream=a)
    for last, now, stream in ((a, b, b), (b, streams.current[0], None), (streams.current[0], a, a)):
        for i, call in enumerate(calls_of(layer, stream)):
            streams.log.clear()
            call()
            waits = streams.log[: streams.log.index(kernels(streams.log)[0])]
            assert (("wait", now.cuda_stream, last.cuda_stream) in waits) == (i == 0 or last is streams.current[0])
            if i == 0:
                for x in (layer.table, layer.lens, layer.ws, layer.rotary.steps):
                    assert ("keep", x.data_ptr(), now.cuda_stream) in streams.log


def test_a_stream_by_its_handle(layer, streams, monkeypatch):
    """A foreign stream may be gone by the next call, so that waits for an event."""
    launched_on(layer, streams, monkeypatch)
    for handle in (0, 4096):
        layer.step(**good(S), stream=handle)
        k = kernels(streams.log)
        assert k and all(e[1:] == (handle, handle) for e in k)
        streams.log.clear()
    layer.step(**good(S))
    assert ("wait", 100, "event of 4096") in streams.log
    streams.log.clear()
    layer.step(**good(S))
    assert not [e for e in streams.log if e[0] == "wait"]


def test_a_larger_workspace_leaves_the_old_one_to_its_streams(layer, streams, monkeypatch):
    launched_on(layer, streams, monkeypatch)
    side = streams.new(55)
    layer.step(**good(S), stream=side)
    old = layer.ws.data_ptr()
    assert ("keep", old, 55) in streams.log
    monkeypatch.setattr(K, "kv_prompt_workspace_bytes", lambda *a: 4096)
    streams.log.clear()
    layer.prompt([5, 0, 2], **good(7), stream=side)
    assert layer.ws.numel() >= 4096 and ("made", 55) in streams.log
    layer.step(**good(S))
    assert ("keep", layer.ws.data_ptr(), 100) in streams.log


def test_an_error_leaves_the_current_stream_as_it_was(layer, streams, monkeypatch):
    launched_on(layer, streams, monkeypatch)
    with pytest.raises(K.KVError):  # more tokens than a slot holds
        layer.prompt([300, 0, 0], **good(300), stream=streams.new(55))
    assert streams.current[-1].cuda_stream == 100


def test_a_handle_may_name_a_new_stream(layer, streams, monkeypatch):
    launched_on(layer, streams, monkeypatch)
    for i in range(2):
        streams.log.clear()
        layer.step(**good(S), stream=4096)
        assert (("wait", 4096, "event of 4096") in streams.log) == (i == 1)
