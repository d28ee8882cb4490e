"""The windowed layer as it is used: chunked prompts, forks, decode steps with
eviction, releases and compaction, every output against attention over the
whole recorded history in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


class History:
    """Each slot's k (rotated, rounded as the pages hold it) and v."""

    def __init__(self, S, Hq, Hkv, d, freqs, window, sinks):
        self.k = [torch.zeros(0, Hkv, d, dtype=torch.float64) for _ in range(S)]
        self.v = [torch.zeros(0, Hkv, d, dtype=torch.float64) for _ in range(S)]
        self.Hq, self.Hkv, self.d, self.f, self.window, self.sinks = Hq, Hkv, d, torch.from_numpy(freqs), window, sinks

    def turn(self, x, pos):  # half layout, rounded to bf16 as the kernel does
        r = len(self.f)
        ang = pos.double().view(-1, 1, 1) * self.f
        a, b = x[..., :r], x[..., r : 2 * r]
        y = torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin(), x[..., 2 * r :]], -1)
        return y.float().to(torch.bfloat16).double()

    def add(self, s, q, k, v):
        n0, n = len(self.k[s]), len(q)
        pos = torch.arange(n0, n0 + n)
        q, k, v = (x.cpu().double().view(n, -1, self.d) for x in (q, k, v))
        self.k[s] = torch.cat([self.k[s], self.turn(k, pos)])
        self.v[s] = torch.cat([self.v[s], v])
        j = torch.arange(n0 + n)
        seen = (j <= pos.view(-1, 1)) & ((j > pos.view(-1, 1) - self.window) | (j < self.sinks))
        x = self.turn(q, pos).view(n, self.Hkv, -1, self.d)
        w = torch.einsum("nhgd,jhd->hgnj", x, self.k[s]) * self.d ** -0.5
        w = torch.softmax(w.masked_fill(~seen, -np.inf), -1)
        out = torch.einsum("hgnj,jhd->nhgd", w, self.v[s]).reshape(n, self.Hq, self.d)
        return out, torch.einsum("hgnj,jhd->nhgd", w, self.v[s].abs()).reshape(n, self.Hq, self.d)


def near(got, want, bound):
    # output and weights rounded to bf16 (2^-8 each); a rounding of q or k that
    # falls the other way moves a score by 2^-8 of a product of two columns:
    # 2^-7 of |score|'s scale on average over d, taken as 2% of the weights
    tol = 2.0 ** -8 * 1.02 * (want.abs() + bound) + 0.02 * bound + 1e-6
    assert ((got.cpu().double() - want).abs() <= tol).all()


@pytest.mark.parametrize("d,window,sinks", [(128, 100, 4), (64, 70, 20)])
def test_chats_as_they_are_used(d, window, sinks):
    from paper_2606_12950_gb300.streaming import WindowedLayer

    S, Hq, Hkv, bs = 6, 8, 2, 16
    freqs = K.kv_rotary_freqs(d, base=10000.0)
    layer = WindowedLayer(160, Hq, Hkv, d, bs, S, 700, window, sinks, freqs)
    h = History(S, Hq, Hkv, d, freqs, window, sinks)
    g = torch.Generator(device="cuda")
    g.manual_seed(d)

    def rows(n):
        x = torch.randn((n, (Hq + 2 * Hkv) * d), generator=g, device="cuda").to(torch.bfloat16)
        return x[:, : Hq * d], x[:, Hq * d : (Hq + Hkv) * d], x[:, (Hq + Hkv) * d :]

    def prompt(counts):
        q, k, v = rows(sum(counts))
        out, at = layer.prompt(counts, q, k, v), 0
        for s, n in enumerate(counts):
            if n:
                near(out[at : at + n], *h.add(s, q[at : at + n], k[at : at + n], v[at : at + n]))
            at += n

    def step():
        q, k, v = rows(S)
        out = layer.step(q, k, v)
        for s in range(S):
            if len(h.k[s]):
                near(out[s : s + 1], *h.add(s, q[s : s + 1], k[s : s + 1], v[s : s + 1]))
            else:
                assert (out[s] == 0).all()

    prompt([250, 0, 3, 0, 0, 0])
    prompt([133, 17, 90, 0, 0, 0])
    for _ in range(20):
        step()
    layer.fork(0, [3, 4])
    for s in (3, 4):
        h.k[s], h.v[s] = h.k[0].clone(), h.v[0].clone()
    for _ in range(40):
        step()
    layer.release(0)
    h.k[0], h.v[0] = h.k[0][:0], h.v[0][:0]
    layer.compact()
    prompt([0, 5, 0, 64, 1, 33])
    for _ in range(20):
        step()
    # what is held: the sinks' blocks and those the next queries can see
    tab, lens = layer.tab.host()
    for s in range(S):
        for b in range(-(-int(lens[s]) // bs)):
            seen = any(j < sinks or j > lens[s] - 1 - window for j in range(b * bs, b * bs + bs))
            assert (tab[s, b] >= 0) == seen
    assert layer.pool.error() == 0
    for s in range(S):
        layer.release(s)
    assert layer.pages_used() == 0
    layer.close()


def test_the_pool_running_out_is_an_error():
    from paper_2606_12950_gb300.streaming import WindowedLayer

    layer = WindowedLayer(4, 4, 2, 64, 16, 2, 200, 32, 0, K.kv_rotary_freqs(64))
    x = torch.zeros((100, 4 * 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(K.KVError) as e:
        layer.prompt([100, 0], x, x, x)
    assert e.value.code == K.KV_ERR_OUT_OF_BLOCKS
    with pytest.raises(ValueError):
        layer.prompt([5], x, x, x)
    layer.close()


def test_the_example_runs(capsys):
    import os
    import subprocess
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "windowed_agents.py"), "--steps", "20",
                        "--prompt", "900", "--chunk", "400", "--window", "256"], capture_output=True, text=True,
                       timeout=200)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "agents" in r.stdout
