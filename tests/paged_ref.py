"""A paged layer's cache with random contents on the GPU, and attention over it
in 64 bits from its definition; test infrastructure only."""
from __future__ import annotations

import numpy as np
import torch

from paper_2606_12950_gb300 import kvpool as K

NAN = float("nan")


class Paged:
    """Sequences of lengths n with nq new tokens each, blocks at random pages of
    a NaN-filled pool.  `held(s, j)` (an array of block indexes -> bool) says
    which blocks exist; the others' table entries are -1.  Rows past a length
    stay NaN."""

    def __init__(self, n, nq, Hq, Hkv, d, bs, seed, held=None, spare=3, max_blocks=None):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.g, self.rng = g, rng
        self.n, self.nq = np.asarray(n, np.int64), np.asarray(nq, np.int64)
        self.S, self.T = len(self.n), int(self.nq.sum())
        self.Hq, self.Hkv, self.d, self.bs = Hq, Hkv, d, bs
        blocks = -(-self.n // bs)
        self.max_blocks = max_blocks or max(1, int(blocks.max()) + 1)
        table = np.full((self.S, self.max_blocks), -1, np.int32)
        want = [(s, j) for s in range(self.S) for j in range(int(blocks[s])) if held is None or held(s, j)]
        pages = len(want) + spare
        ids = rng.permutation(pages)
        for (s, j), i in zip(want, ids):
            table[s, j] = i
        self.host_table = table
        self.pool = torch.full((pages, 2, Hkv, bs, d), NAN, dtype=torch.bfloat16, device="cuda")
        for s, j in want:
            m = int(min(bs, self.n[s] - j * bs))
            self.pool[table[s, j], :, :, :m] = self.normal(2, Hkv, m, d)
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.h = K.kv_pool_create(self.pool, self.pool.numel() * 2, bs, [(Hkv, d)], self.err)
        self.table = torch.from_numpy(table).cuda()
        self.lens = torch.from_numpy(self.n.astype(np.int32)).cuda()
        self.starts_host = np.concatenate([[0], np.cumsum(self.nq)])
        self.starts = torch.from_numpy(self.starts_host.astype(np.int32)).cuda()

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32).to(torch.bfloat16)

    def error(self):
        return K.kv_pool_get_error(self.h, None)

    def close(self):
        torch.cuda.synchronize()
        K.kv_pool_destroy(self.h)

    def reference(self, q, scale, window, sinks):
        """(out, bound) [T, Hq, d] in float64 on the host: each query at position
        p of its sequence over j <= p with j > p - window or j < sinks; zeros at
        p < 0.  bound: sum of weight * |v|, by which rounded weights can move
        out.  Rows of V with an infinity or a NaN count where they are seen."""
        out = torch.zeros(self.T, self.Hq, self.d, dtype=torch.float64)
        bound = torch.zeros_like(out)
        G = self.Hq // self.Hkv
        pool, q = self.pool.cpu(), q.cpu().double()
        for s in range(self.S):
            nq, n = int(self.nq[s]), int(self.n[s])
            p = torch.arange(n - nq, n).clamp(min=-1)
            if nq == 0 or n == 0:
                continue
            j = torch.arange(n)
            seen = j <= p.view(-1, 1)
            if window:
                seen &= (j > p.view(-1, 1) - window) | (j < sinks)
            j = j[seen.any(0)]
            seen = seen[:, j]
            blk = torch.from_numpy(self.host_table[s].astype(np.int64))[j // self.bs]
            assert (blk >= 0).all()
            k, v = pool[blk, :, :, j % self.bs].double().permute(1, 2, 0, 3)  # [Hkv, keys, d]
            rows = slice(int(self.starts_host[s]), int(self.starts_host[s]) + nq)
            x = q[rows].view(nq, self.Hkv, G, self.d).permute(1, 2, 0, 3)
            x = (x @ k.unsqueeze(1).transpose(2, 3) * scale).masked_fill(~seen, -np.inf)
            w = torch.softmax(x, -1)
            odd = ~torch.isfinite(v).all(2).all(0)  # tokens: their products stay apart from unseen weights
            w[..., p < 0, :] = 0
            o = w @ torch.where(odd.view(1, -1, 1), 0.0, v).unsqueeze(1)
            for i in odd.nonzero().flatten().tolist():
                o = o + torch.where(seen[:, i].view(1, 1, -1, 1), w[..., i : i + 1] * v[:, i].view(self.Hkv, 1, 1, -1), 0.0)
            bnd = w @ torch.where(odd.view(1, -1, 1), 0.0, v).abs().unsqueeze(1)
            out[rows] = o.permute(2, 0, 1, 3).reshape(nq, self.Hq, self.d)
            bound[rows] = bnd.permute(2, 0, 1, 3).reshape(nq, self.Hq, self.d)
        return out.cuda(), bound.cuda()


def check(out, ref, bound):
    """Output rounding is at most 2^-8 of the value, and so is that of each
    weight before P.V: 2^-8 (|ref| + sum w |v|), and 2% and 1e-6 for the fp32
    sums and the 2^x approximation (below 2^-20 each)."""
    out = out.double().view(ref.shape)
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(out), nan)
    inf = torch.isinf(ref)
    assert torch.equal(out[inf], ref[inf])
    ok = ~(nan | inf)
    tol = 2.0 ** -8 * 1.02 * (ref.abs() + bound.nan_to_num(posinf=0.0)) + 1e-6
    worst = ((out - ref).abs() - tol)[ok]
    assert worst.numel() == 0 or worst.max().item() <= 0, worst.max().item()


def holds(n, nq, window, sinks, bs):
    """Blocks that some query sees, for Paged(held=)."""
    def held(s, j):
        lo = max(0, int(n[s]) - max(1, int(nq[s])) - window + 1)
        return j * bs < sinks or (j + 1) * bs > lo
    return held if window else None
