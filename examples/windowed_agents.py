"""Agents over one long task: a prompt read in chunks, forked into agents that
go on by themselves, each over a sliding window with sinks.

    python examples/windowed_agents.py [--agents 12] [--prompt 6000] [--steps 400]

Prints what the pages, the prompt and the decode steps come to on this GPU.
Inputs are random: the layer's projections are not part of this library.
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2606_12950_gb300 import kvpool as K  # noqa: E402
from paper_2606_12950_gb300.runner import VmmPool  # noqa: E402
from paper_2606_12950_gb300.streaming import WindowedLayer  # noqa: E402


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--agents", type=int, default=12)
    ap.add_argument("--prompt", type=int, default=6000)
    ap.add_argument("--chunk", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=400)
    ap.add_argument("--window", type=int, default=1024)
    ap.add_argument("--sinks", type=int, default=4)
    a = ap.parse_args()
    Hq, Hkv, d, bs = 32, 8, 128, 16
    freqs = K.kv_rotary_freqs(d, base=500000.0, scaling=K.KV_ROTARY_BY_PARTS, factor=4.0, original_len=8192)
    most = a.prompt + a.steps + 1
    # virtual room for every agent's whole run; physical memory follows the pages held
    page = 2 * Hkv * bs * d * 2
    pool = VmmPool((a.agents + 1) * -(-most // bs) * page + (64 << 20), page, bs, [(Hkv, d)])
    layer = WindowedLayer(0, Hq, Hkv, d, bs, a.agents + 1, most, a.window, a.sinks, freqs, pool=pool)
    g = torch.Generator(device="cuda")
    g.manual_seed(0)

    def rows(n):  # of one fused projection: q, k and v are column ranges
        x = torch.randn((n, (Hq + 2 * Hkv) * d), generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)
        return x[:, : Hq * d], x[:, Hq * d : (Hq + Hkv) * d], x[:, (Hq + Hkv) * d :]

    def clock(f):
        torch.cuda.synchronize()
        t = time.perf_counter()
        f()
        torch.cuda.synchronize()
        return time.perf_counter() - t

    def mapped():
        return f"{layer.pages_used()} pages, {pool.stats()['bytes_mapped'] / 2**20:.0f} MiB mapped"

    def read_prompt():
        for at in range(0, a.prompt, a.chunk):
            n = min(a.chunk, a.prompt - at)
            layer.prompt([n] + [0] * a.agents, *rows(n))

    clock(read_prompt)  # the first pass loads the kernels
    layer.release(0)
    t = clock(read_prompt)
    print(f"prompt: {a.prompt} tokens in {t * 1e3:.2f} ms; {mapped()} of {-(-a.prompt // bs)} pages written "
          f"(window {a.window}, {a.sinks} sinks)")
    layer.fork(0, list(range(1, a.agents + 1)))
    layer.release(0)
    print(f"forked into {a.agents} agents: {mapped()}")

    def decode():
        for _ in range(a.steps):
            layer.step(*rows(a.agents + 1))

    t = clock(decode)
    print(f"decode: {a.steps} steps of {a.agents} agents, {t / a.steps * 1e6:.1f} us a step; {mapped()}")
    for s in range(1, a.agents + 1, 2):
        layer.release(s)
    moved = layer.compact()
    print(f"half the agents done, {moved} pages moved: {mapped()}")
    assert pool.error() == 0
    layer.close()
    pool.close()


if __name__ == "__main__":
    main()
