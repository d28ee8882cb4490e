"""The packed layer over an elastic pool with a limit: it packs as far as there is
memory, and outputs and cache are right wherever a token lies."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_12950_gb300 import kvpool as K  # noqa: E402

pytestmark = pytest.mark.gpu


def test_a_pool_with_a_limit():
    from paper_2606_12950_gb300.runner import VmmPool
    from paper_2606_12950_gb300.streaming import PackedLayer
    from tests.test_packed_layer_gpu import Chats, near

    S, Hq, Hkv, d, bs, keep = 3, 16, 8, 128, 64, 1
    block = 2 * Hkv * bs * d * 2                    # 256 KB: eight a chunk of 2 MB
    pool = VmmPool(512 * block, block // 32, bs, [(Hkv, d), (Hkv, d | K.KV_Q4)], physical_limit=24 * block)
    pool.buf = pool.pages.view(-1)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)

    freqs = K.kv_rotary_freqs(d)
    wq, wk = (1 + 0.3 * normal(2, d).float()).to(torch.bfloat16)
    layer = PackedLayer(0, Hq, Hkv, d, bs, S, 3000, keep, freqs, norm=K.HeadNorm(wq, wk, 1e-5), pool=pool)
    chats = Chats(layer, freqs, wq, wk, 1e-5)

    def rows(n):
        x = normal(n, (Hq + 2 * Hkv) * d)
        return x[:, : Hq * d], x[:, Hq * d : (Hq + Hkv) * d], x[:, (Hq + Hkv) * d :]

    def prompt(counts):
        q, k, v = rows(sum(counts))
        at, want = 0, []
        for s, n in enumerate(counts):
            if n:
                r = slice(at, at + n)
                want.append((r, *chats.expect(s, q[r], k[r], v[r])))
                at += n
        out = layer.prompt(counts, q, k, v)
        torch.cuda.synchronize()
        for r, o, a in want:
            near(out[r], o, a)

    def step():
        q, k, v = rows(S)
        want = {s: chats.expect(s, q[s : s + 1], k[s : s + 1], v[s : s + 1]) for s in np.nonzero(layer.tab.lens())[0]}
        out = layer.step(q, k, v)
        torch.cuda.synchronize()
        for s, w in want.items():
            near(out[s : s + 1], *w)

    # 24 pages: all that may be mapped, in bf16
    prompt([20 * bs - 7, 3 * bs, bs - 3])
    assert layer.tab4.lens().tolist() == [0, 0, 0] and pool.stats()["bytes_mapped"] == 24 * block
    layer.release(1)                                # three pages: room for nine packed ones
    chats.k[1], chats.v[1] = chats.k[1][:0], chats.v[1][:0]
    for _ in range(3):
        step()
    n = layer.tab.lens()
    assert n[0] == 20 * bs - 4 and layer.tab4.lens()[0] == 19 * bs  # and those that they freed
    for _ in range(10):
        step()
    for s in (0, 2):
        chats.check_cache(s)
    prompt([0, 5 * bs, 0])
    step()
    for s in range(S):
        chats.check_cache(s)
    assert pool.stats()["bytes_mapped"] <= 24 * block and pool.error() == 0
    layer.close()
    pool.close()
