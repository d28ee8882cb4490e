"""The windowed layer on streams other than the default one: late inputs, memory
that is used again at once, calls that change streams.  The bits are those of the
same calls on the default stream."""
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu

S, HQ, HKV, D, BS = 5, 8, 2, 128, 16
LATE = 2_000_000  # clocks of an idle kernel, about a millisecond


def script():
    """(call, arguments) of a small server's day."""
    yield "prompt", [600, 0, 3, 0, 0]
    yield "prompt", [200, 40, 90, 0, 0]
    for _ in range(5):
        yield "step", None
    yield "fork", (0, [3, 4])
    for _ in range(5):
        yield "step", None
    yield "release", 0
    yield "compact", None
    yield "prompt", [5, 64, 0, 1, 33]
    for _ in range(3):
        yield "step", None


def run(streams, around=None, window=100):
    """The script's results; streams(i) is call i's stream, `around` torch's
    current one."""
    from paper_2606_12950_gb300.streaming import WindowedLayer

    torch.cuda.synchronize()
    outs = []
    with torch.cuda.stream(around if around is not None else torch.cuda.default_stream()):
        layer = WindowedLayer(120, HQ, HKV, D, BS, S, 1000, window, 4, K.kv_rotary_freqs(D))
        gen = torch.Generator().manual_seed(3)
        for i, (what, a) in enumerate(script()):
            stream = streams(i)
            if what == "release":
                layer.release(a)
                continue
            if what == "fork":
                layer.fork(*a, stream=stream)
                continue
            if what == "compact":
                layer.compact(stream=stream)
                continue
            n = sum(a) if what == "prompt" else S
            host = torch.randn((n, (HQ + 2 * HKV) * D), generator=gen).to(torch.bfloat16).pin_memory()
            x = torch.full(host.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
            torch.cuda._sleep(LATE)  # the rows come late on the current stream
            x.copy_(host, non_blocking=True)
            q, k, v = x[:, : HQ * D], x[:, HQ * D : (HQ + HKV) * D], x[:, (HQ + HKV) * D :]
            side = layer.last if stream is None else torch.cuda.ExternalStream(getattr(stream, "cuda_stream", stream))
            if stream is not None:
                with torch.cuda.stream(side):
                    torch.cuda._sleep(LATE)  # and the call's own stream is busy
            out = layer.prompt(a, q, k, v, stream=stream) if what == "prompt" else layer.step(q, k, v, stream=stream)
            del x, q, k, v
            # what the call and its caller gave back is taken and written at once
            trash = [torch.full((n, w * D), float("nan"), dtype=torch.bfloat16, device="cuda")
                     for w in (HQ + 2 * HKV, HQ, HQ)]
            trash.append(torch.full((S + 1,), 2 ** 30, dtype=torch.int32, device="cuda"))
            trash.append(torch.full((layer.ws.numel(),), 255, dtype=torch.uint8, device="cuda"))
            if stream is not None:
                torch.cuda.current_stream().wait_stream(side)
            outs.append(out.clone())
            del trash
        torch.cuda.synchronize()
        assert layer.pool.error() == 0
        layer.close()
    return outs


@pytest.fixture(scope="module")
def want():
    out = run(lambda i: None)
    assert all(torch.isfinite(x).all() for x in out)
    return out


def same(got, want):
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_current_stream_when_it_is_not_the_default(want):
    same(run(lambda i: None, around=torch.cuda.Stream()), want)


def test_a_stream_beside_the_current_one(want):
    st = torch.cuda.Stream()
    same(run(lambda i: st), want)
    same(run(lambda i: st, around=torch.cuda.Stream()), want)


def test_calls_that_change_streams(want):
    sts = [torch.cuda.Stream(), torch.cuda.Stream(), None]
    same(run(lambda i: sts[i % 3]), want)
    same(run(lambda i: sts[i * 7 % 3], around=torch.cuda.Stream()), want)


def test_streams_by_their_handles(want):
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    hs = [a.cuda_stream, b.cuda_stream, None, 0]
    same(run(lambda i: hs[i % 4], around=torch.cuda.Stream()), want)
