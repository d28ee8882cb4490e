"""A paged cache whose older tokens are held in 4 bits, with random contents on
the GPU, the packed format read back from its bytes, and attention over it in 64
bits; test infrastructure only."""
from __future__ import annotations

import numpy as np
import torch

from paper_2606_12950_gb300 import kvpool as K

GROUP = 64


def quantised(x):
    """(codes, s, z) of rows x [..., d] (bf16 values) in groups of 64 columns, by
    the definition: s from fp32 arithmetic, the codes in 64 bits."""
    x = x.float().unflatten(-1, (-1, GROUP))
    z, top = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)  # (both NaN where a value is)
    span = top - z
    s = (span / 15.0).to(torch.bfloat16).float()
    s = torch.where(s >= 2.0 ** -100, s, 0.0)
    s = torch.where(span < 2.0 ** 80, s, float("nan"))
    q = (x - z).double() / torch.where(s > 0, s, 1.0).double()
    codes = torch.where(s > 0, torch.round(q), 0.0).nan_to_num(0.0)
    return codes, s, z


def values(x):
    """What rows x stand for once packed, in 64 bits."""
    c, s, z = quantised(x)
    return (c * s.double() + z.double()).flatten(-2)


def parse_block(raw, Hkv, bs, d):
    """(codes, s, z) of a packed block's bytes, [2, Hkv, bs, d / 64, 64 or 1]."""
    NG, tile = d // 64, 18 * d
    t = np.frombuffer(raw.tobytes(), np.uint8)[: Hkv * (bs // 16) * tile].reshape(Hkv, bs // 16, tile)
    codes = np.zeros((2, Hkv, bs // 16, 16, d), np.uint8)
    par = np.zeros((2, Hkv, bs // 16, 16, NG, 2), np.float32)
    k = t[:, :, : 8 * d].copy().view(np.uint32).reshape(Hkv, -1, 16, 4, d // 32)  # [row, t, word]
    v = t[:, :, 8 * d : 16 * d].copy().view(np.uint32).reshape(Hkv, -1, NG, 8, 4, 4)  # [v, g, t, word]
    for j in range(d // 32):
        for lane in range(4):
            for i in range(8):
                codes[0, :, :, :, 64 * (j // 2) + 32 * (j % 2) + 8 * lane + i] = (k[:, :, :, lane, j] >> (4 * i)) & 15
    place = [(0, 0), (0, 1), (8, 0), (8, 1), (1, 0), (1, 1), (9, 0), (9, 1)]  # of a nibble: token, column
    for c in range(NG):
        for g in range(8):
            for lane in range(4):
                for m in range(4):
                    for i, (tok, col) in enumerate(place):
                        codes[1, :, :, 2 * lane + tok, 64 * c + 8 * g + 2 * m + col] = (v[:, :, c, g, lane, m] >> (4 * i)) & 15
    for kv in (0, 1):
        w = t[:, :, 16 * d :].copy().view(np.uint32).reshape(Hkv, -1, 16, 2, NG)[:, :, :, kv]
        par[kv, ..., 0] = (w << 16).view(np.float32)
        par[kv, ..., 1] = (w & 0xFFFF0000).view(np.float32)
    shape = (2, Hkv, bs, NG)
    return codes.reshape(*shape, 64), par[..., 0].reshape(*shape, 1), par[..., 1].reshape(*shape, 1)


class PagedQ4:
    """Sequences of lengths n (post-append where `append`), the first p of each
    in 4 bits, at random blocks of one pool of both kinds; unused bytes are NaN
    patterns.  make(kv, seq, tokens) -> bf16 [Hkv, tokens, d] gives the rows."""

    def __init__(self, n, p, Hq, Hkv, d, bs, seed, append=True, make=None, extra=2, fill=0xFF):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.g = g
        self.n, self.p = np.asarray(n, np.int64), np.asarray(p, np.int64)
        self.S, self.Hq, self.Hkv, self.d, self.bs = len(self.n), Hq, Hkv, d, bs
        make = make or (lambda kv, s, m: self.normal(Hkv, m, d))
        b4, b16 = self.p // bs, -(-self.n // bs)
        self.max_blocks, self.max_blocks4 = max(1, int(b16.max()) + 1), max(1, int(b4.max()) + 1)
        n4, held = int(b4.sum()), [(s, j) for s in range(self.S) for j in range(int(b4[s]), int(b16[s]))]
        n16 = len(held) + extra
        self.block = 2 * Hkv * bs * d * 2
        total = n16 + max(1, n4) + -(-n4 // 3) + 1
        self.buf = torch.full((total * self.block,), fill, dtype=torch.uint8, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.h = K.kv_pool_create(self.buf, self.buf.numel(), bs, [(Hkv, d), (Hkv, d | K.KV_Q4)], self.err,
                                  page_bytes=self.block // 32, shuffle_seed=seed + 1)
        ids16 = K.kv_alloc_blocks(self.h, 0, n16)
        self.rows = []  # bf16 [2, Hkv, n, d] of each sequence, on the device
        t16, t4 = np.full((self.S, self.max_blocks), -1, np.int32), np.full((self.S, self.max_blocks4), -1, np.int32)
        for (s, j), i in zip(held, rng.permutation(ids16)):
            t16[s, j] = i
        ids4 = rng.permutation(K.kv_alloc_blocks(self.h, 1, n4)) if n4 else np.zeros(0, np.int32)
        tmp = K.kv_alloc_blocks(self.h, 0, n4) if n4 else ids4
        k = 0
        for s in range(self.S):
            x = torch.stack([make(kv, s, int(self.n[s])) for kv in (0, 1)]) if self.n[s] else torch.zeros(
                (2, Hkv, 0, d), dtype=torch.bfloat16, device="cuda")
            self.rows.append(x)
            for j in range(int(b16[s])):
                m = int(min(bs, self.n[s] - j * bs, self.n[s] - append - j * bs))
                part = x[:, :, j * bs : j * bs + m]
                if j < b4[s]:
                    t4[s, j] = ids4[k]
                    self.block16(tmp[k])[:] = part
                    k += 1
                elif m > 0:
                    self.block16(t16[s, j])[:, :, :m] = part
        if n4:
            K.kv_pack_blocks(self.h, 0, 1, tmp, ids4)
            torch.cuda.synchronize()
            for i in tmp:
                self.buf[int(i) * self.block // 32 :][: self.block] = fill
            K.kv_free_blocks(self.h, 0, tmp)
        self.host_table, self.host_table4 = t16, t4
        self.table, self.table4 = torch.from_numpy(t16).cuda(), torch.from_numpy(t4).cuda()
        self.lens = torch.from_numpy(self.n.astype(np.int32)).cuda()
        self.packed = torch.from_numpy(self.p.astype(np.int32)).cuda()
        self.k_new = self.v_new = None
        if append:
            self.k_new, self.v_new = (torch.stack([x[kv, :, -1] if x.shape[2] else torch.zeros(Hkv, d, device="cuda").to(x)
                                                   for x in self.rows]).contiguous() for kv in (0, 1))
        n_ws = K.kv_q4_workspace_bytes(self.h, 1, self.S, Hq, self.max_blocks)
        self.ws = torch.full((max(256, n_ws),), 0xFF, dtype=torch.uint8, device="cuda")

    def block16(self, i):
        return self.buf[int(i) * self.block // 32 :][: self.block].view(torch.bfloat16).view(2, self.Hkv, self.bs, self.d)

    def raw4(self, i):
        return self.buf[int(i) * self.block // 32 :][: self.block * 9 // 32].cpu().numpy()

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32).to(torch.bfloat16)

    def run(self, q, scale, out=None, stream=None):
        out = torch.full((self.S, self.Hq, self.d), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
        K.paged_decode_attn_q4(self.h, 0, 1, q, self.k_new, self.v_new, out, self.table, self.lens, self.max_blocks,
                               self.table4, self.packed, self.max_blocks4, self.S, self.Hq, scale, self.ws,
                               self.ws.numel(), stream)
        return out

    def reference(self, q, scale):
        """(out, tol) [S, Hq, d] in float64.  tol: the output's rounding to bf16,
        2^-8 of the value; weights rounded to fp16 with V's scale, 2^-11 of p s c
        each (2% for what is below), and to bf16 before bf16 rows, 2^-8; 2^-14 of
        sum p |v| for the scores' fp32 sums, whose terms add to under 64 here (2^-24
        of that some times over, in both weights and their sum) and 2^x."""
        G = self.Hq // self.Hkv
        out = torch.zeros(self.S, self.Hq, self.d, dtype=torch.float64, device="cuda")
        tol = torch.zeros_like(out)
        for s in range(self.S):
            n, p = int(self.n[s]), int(self.p[s])
            if n == 0:
                continue
            x = self.rows[s]
            c, sc, z = quantised(x[:, :, :p])
            k, v = torch.cat([values(x[:, :, :p]), x[:, :, p:].double()], 2)
            sc_c = torch.cat([(c * sc.double()).flatten(-2)[1], torch.zeros_like(v[:, p:])], 1)
            mag = torch.cat([(c * sc.double() + z.abs().double()).flatten(-2)[1], v[:, p:].abs()], 1)
            w = torch.softmax(q[s].view(self.Hkv, G, self.d).double() @ k.transpose(1, 2) * scale, -1)
            o = w @ v
            t = 2.0 ** -8 * 1.02 * o.abs() + 2.0 ** -11 * 1.02 * (w @ sc_c) + 2.0 ** -14 * (w @ mag)
            t += 2.0 ** -8 * 1.02 * (w[..., p:] @ v[:, p:].abs())
            out[s], tol[s] = o.reshape(self.Hq, self.d), t.reshape(self.Hq, self.d)
        return out, tol + 1e-30

    def error(self):
        return K.kv_pool_get_error(self.h, None)

    def close(self):
        torch.cuda.synchronize()
        K.kv_pool_destroy(self.h)


def check(out, ref, tol):
    out = out.double()
    assert torch.equal(torch.isnan(out), torch.isnan(ref))
    fine = ~torch.isnan(ref)
    over = ((out - ref).abs() - tol)[fine]
    assert over.numel() == 0 or over.max().item() <= 0, (over.max().item(), ((out - ref).abs() / tol)[fine].max().item())
