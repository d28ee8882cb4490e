"""The operators of a layer with normed heads and a cache held in 4 bits, as
measurable cases.

One pass is one call (pack: two) on one layer:

  norm     the new tokens' q and k normed for each head, rotated to their
           positions, k and v written into the bf16 cache: one token a
           sequence, or ragged prompt chunks
  pack     full bf16 blocks packed into 4 bits, and read back
  unpack   blocks held in 4 bits written out in bf16
  decode   one query a sequence over its context: the older tokens in 4 bits,
           the last ones in bf16 blocks, the step's new K/V row appended in the
           same call

A group of 4 bits is 64 columns of a token's head: code c in 0..15 stands for
s c + z, z the group's least value, s = (greatest - z) / 15 rounded to bf16,
c the nearest code, ties to even.

A case's lengths are the quantiles of its distribution, so that its work
depends on the case alone; the seed sets their order, where the blocks lie and
all values.  Passes do not advance the lengths, so they can be repeated.
"""
from __future__ import annotations

import math
from statistics import NormalDist

import numpy as np
import torch

own = False

GROUP = 64  # columns that share a scale


def _case(name, op, seqs, heads, *, head_dim=128, block=16, ctx="uniform", lo=0, hi=0, q_lo=1, q_hi=1, keep=0, rot=0,
          interleaved=False, offset=0.0):
    """heads: query x KV heads.  ctx, lo, hi: cached tokens before the call.
    q_lo, q_hi: the call's new tokens a sequence.  keep: the last tokens that
    stay in bf16, at least.  rot: rotated columns of a head; offset: added to
    the norms' weights.  pack, unpack: seqs blocks."""
    c = {"op": op, "seqs": seqs, "heads": heads, "head_dim": head_dim, "block": block, "ctx": ctx, "lo": lo, "hi": hi,
         "q_lo": q_lo, "q_hi": q_hi, "keep": keep, "rot": rot, "interleaved": interleaved, "offset": offset}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest model of the tests, a step of four short chats
        _case("norm_tiny_step", "norm", 4, "4x2", head_dim=64, lo=17, hi=255, rot=64),
        # an ordinary decode batch's step: rows of one fused projection
        _case("norm_step", "norm", 64, "32x8", ctx="lognormal", lo=1024, hi=16384, rot=128),
        # admitted prompts late in long contexts, half of each head rotated in
        # adjacent pairs
        _case("norm_prompts", "norm", 24, "40x8", lo=5, hi=60000, q_lo=3, q_hi=1333, rot=64, interleaved=True,
              offset=1.0),
        # the blocks that a step of a small batch has filled
        _case("pack_step", "pack", 5, "32x8"),
        # the prompts of a batch packed after they were read
        _case("pack_prompts", "pack", 4000, "32x8"),
        # a chat that goes on with a new prompt
        _case("unpack_chat", "unpack", 130, "16x16", head_dim=64, block=32),
        # a batch of long chats that go on
        _case("unpack_batch", "unpack", 6000, "32x8"),
        # the smallest model of the tests, four short chats
        _case("decode_tiny", "decode", 4, "4x2", head_dim=64, lo=17, hi=255, keep=1),
        # one user's long document
        _case("decode_document", "decode", 1, "32x8", lo=100000, hi=100000, keep=64),
        # an ordinary batch
        _case("decode_batch", "decode", 64, "32x8", ctx="lognormal", lo=1024, hi=16384, keep=16),
        # a large batch of contexts of all lengths, pages of 32 tokens
        _case("decode_many", "decode", 250, "40x8", block=32, ctx="pareto", lo=900, hi=12000, keep=33),
        # a small model without grouped heads
        _case("decode_single_heads", "decode", 40, "16x16", head_dim=64, block=32, lo=0, hi=6000, keep=1),
    ]


# no drawn case costs more than the largest listed one of its kind
_MOST = {"norm": 4.2e8, "pack": 6.0e8, "unpack": 5.0e8, "decode": 6.0e8}


def draw(rng):
    """A case of the same ranges."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["norm", "norm", "pack", "unpack", "decode", "decode", "decode"])
    head_dim, block = rng.choice([64, 128, 128]), rng.choice([16, 16, 32, 48, 64])
    kv = rng.choice([2, 4, 8, 8, 16])
    heads = "%dx%d" % (kv * rng.choice([1, 2, 4, 4, 5, 8]), kv)
    ctx = rng.choice(["uniform", "lognormal", "pareto"])
    common = dict(head_dim=head_dim, block=block, ctx=ctx)
    if op == "norm":
        q_hi = rng.choice([1, log_int(2, 4000)])
        c = _case("", op, log_int(1, 400), heads, lo=rng.randrange(0, 400), hi=log_int(400, 100000), q_lo=1, q_hi=q_hi,
                  rot=rng.choice([16, 32, 64, head_dim, head_dim]), interleaved=rng.random() < 0.5,
                  offset=rng.choice([0.0, 1.0]), **common)
    elif op == "decode":
        c = _case("", op, log_int(1, 400), heads, lo=rng.randrange(0, 900), hi=log_int(900, 120000),
                  keep=log_int(1, 300), **common)
    else:
        c = _case("", op, log_int(1, 6000), heads, head_dim=head_dim, block=block)
    while work(c)["bytes"] > _MOST[op] or _footprint(c) > 3.0e10:
        if c["seqs"] > 1:
            c["seqs"] = c["seqs"] * 3 // 4
        else:
            c["q_hi"] = max(1, c["q_hi"] * 3 // 4)
            c["hi"] = max(c["lo"], c["hi"] * 3 // 4)
    return c


# ------------------------------------------------------------- the sizes ---
def _heads(c):
    return tuple(int(x) for x in c["heads"].split("x"))


def _quantiles(kind, lo, hi, n):
    """n quantiles, smallest first; lognormal about max(lo, hi / 8)."""
    u = (np.arange(n) + 0.5) / n
    hi = max(hi, lo)
    if kind == "lognormal":
        x = np.clip(max(lo, hi / 8) * np.exp([NormalDist().inv_cdf(v) for v in u]), min(lo, 16), hi)
    elif kind == "pareto":  # bounded, exponent 1.2
        a = max(1, lo)
        x = a / np.power(1.0 - u * (1.0 - (a / max(a, hi)) ** 1.2), 1 / 1.2)
    else:
        x = lo + u * (hi - lo)
    return np.floor(x).astype(np.int64)


def _sizes(c):
    """New tokens and lengths (with them) of the sequences, in a fixed order."""
    nq = _quantiles("uniform", c["q_lo"], c["q_hi"] + 1 if c["q_hi"] > c["q_lo"] else c["q_hi"], c["seqs"])
    nq = np.minimum(nq, c["q_hi"])
    ctx = np.random.default_rng(7).permutation(_quantiles(c["ctx"], c["lo"], c["hi"], c["seqs"]))
    return nq, ctx + nq


def _packed(c, n):
    """Tokens held in 4 bits: the full blocks before the last `keep` tokens."""
    return np.maximum(0, n - c["keep"]) // c["block"] * c["block"]


def work(c):
    Hq, Hkv = _heads(c)
    d = c["head_dim"]
    full, packed = 2 * d, d // 2 + d // GROUP * 4  # bytes of a head's row in bf16 and in 4 bits
    if c["op"] in ("pack", "unpack"):
        rows = c["seqs"] * c["block"] * 2 * Hkv
        return {"bytes": rows * (full + packed) * (2 if c["op"] == "pack" else 1), "flops": rows * d * 4}
    nq, n = _sizes(c)
    T = int(nq.sum())
    if c["op"] == "norm":
        return {"bytes": T * 2 * (Hq + 2 * Hkv) * full, "flops": T * (Hq + Hkv) * (d * 4 + c["rot"] * 3)}
    old = _packed(c, n)
    byts = int(old.sum()) * 2 * Hkv * packed + int((n - old).sum()) * 2 * Hkv * full  # the new row is written, not read
    return {"bytes": byts + T * (2 * Hq + 2 * Hkv) * full, "flops": int(n.sum()) * Hq * d * 4}


def _footprint(c):
    """About what the plain form holds at its largest."""
    Hq, Hkv = _heads(c)
    nq, n = _sizes(c)
    if c["op"] == "norm":
        return int(nq.sum()) * Hq * c["head_dim"] * 32
    if c["op"] == "decode":
        return c["seqs"] * int(n.max()) * Hkv * c["head_dim"] * 12
    return c["seqs"] * c["block"] * 2 * Hkv * c["head_dim"] * 24


# ------------------------------------------------------------- the state ---
class _State:
    handle = None

    def __del__(self):
        if self.handle:
            self.K.kv_pool_destroy(self.handle)


def prepare(case, seed):
    st = _State()
    st.case = c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    (Hq, Hkv), d, bs, S = _heads(c), c["head_dim"], c["block"], c["seqs"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)

    n4 = S if c["op"] in ("pack", "unpack") else 0  # blocks held in 4 bits
    if n4:
        n_bf16 = (2 if c["op"] == "pack" else 1) * S
        order = torch.from_numpy(rng.permutation(n_bf16)).cuda()
        st.src, st.dst = order[:S], order[-S:]
    else:
        nq, n = _sizes(c)
        order = rng.permutation(S)
        nq, n = nq[order], n[order]
        old = _packed(c, n) if c["op"] == "decode" else n - nq  # not in bf16 blocks, or not touched
        st.max_len, st.T = int(n.max()), int(nq.sum())
        st.max_blocks = max(1, -(-st.max_len // bs))
        at = np.arange(st.max_blocks)
        held = (at < -(-n // bs)[:, None]) & (at >= (old // bs)[:, None])
        n_held = int(held.sum())
        n_bf16 = n_held + n_held // 9 + 8
        table = np.full(held.shape, -1, dtype=np.int32)
        table[held] = rng.permutation(n_bf16)[:n_held]
        st.table = torch.from_numpy(table).cuda()
        st.lens = torch.from_numpy(n.astype(np.int32)).cuda()
        st.starts = torch.from_numpy(np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)).cuda()
        st.scale = d ** -0.5
        if c["op"] == "decode":
            n4 = int(old.sum()) // bs
            table = np.full(held.shape, -1, dtype=np.int32)
            table[at < (old // bs)[:, None]] = rng.permutation(n4)
            st.table4 = torch.from_numpy(table).cuda()
            st.lens4 = torch.from_numpy(old.astype(np.int32)).cuda()
    # a K channel in sixteen is an outlier, as keys have them
    channel = torch.ones(2, Hkv, 1, d, device="cuda", dtype=torch.bfloat16)
    channel[0, :, :, torch.from_numpy(rng.permutation(d)[: d // 16]).cuda()] = 4.0
    st.pages = normal(n_bf16, 2, Hkv, bs, d) * channel
    if c["op"] == "norm":
        qkv = normal(st.T, (Hq + 2 * Hkv) * d) * 3.0  # rows of one fused projection
        st.q, st.k, st.v = qkv[:, : Hq * d], qkv[:, Hq * d : (Hq + Hkv) * d], qkv[:, (Hq + Hkv) * d :]
        st.q_out = torch.empty(st.T, Hq, d, device="cuda", dtype=torch.bfloat16)
        st.q_weight, st.k_weight = normal(d) * 0.3 + (1.0 - c["offset"]), normal(d) * 0.3 + (1.0 - c["offset"])
        st.eps = 1e-6
        st.freqs = 500000.0 ** (-2.0 * np.arange(c["rot"] // 2) / c["rot"])
    elif c["op"] == "decode":
        st.q, st.k, st.v = normal(S, Hq, d), normal(S, Hkv, d) * channel[0].view(Hkv, d), normal(S, Hkv, d)
        st.out = torch.empty(S, Hq, d, device="cuda", dtype=torch.bfloat16)
    if c["op"] in ("unpack", "decode"):  # what the 4-bit blocks were packed from
        st.old = normal(n4, 2, Hkv, bs, d) * channel
    if own:  # the pool's handle and what its calls keep
        _open(st, n4)
    elif c["op"] in ("unpack", "decode"):
        st.codes, st.scales, st.least = _quantise(st.old)
    return st


def _open(st, n4):
    from paper_2606_12950_gb300 import kvpool as K

    st.K, c = K, st.case
    (Hq, Hkv), d, bs, n = _heads(c), c["head_dim"], c["block"], len(st.pages)
    st.err = torch.zeros(1, dtype=torch.int32, device="cuda")
    if c["op"] == "norm":
        st.handle = K.kv_pool_create(st.pages, st.pages.numel() * 2, bs, [(Hkv, d)], st.err)
        K.kv_alloc_blocks(st.handle, 0, n)
        st.steps = torch.from_numpy(K.kv_rotary_steps(st.freqs).view(np.int64)).cuda()
        st.rotary = K.Rotary(c["rot"], st.steps, interleaved=c["interleaved"])
        st.norm = K.HeadNorm(st.q_weight, st.k_weight, eps=st.eps, offset=c["offset"])
        return
    # one pool of both kinds of block: 32 pages a bf16 block, 9 a 4-bit one, three of which share 32 pages
    old = st.old if c["op"] in ("unpack", "decode") else st.pages[:0]
    block = 2 * Hkv * bs * d * 2
    buf = torch.empty((n + len(old) + -(-n4 // 3)) * block // 2, dtype=torch.bfloat16, device="cuda")
    st.handle = K.kv_pool_create(buf, buf.numel() * 2, bs, [(Hkv, d), (Hkv, d | K.KV_Q4)], st.err, page_bytes=block // 32)
    ids = K.kv_alloc_blocks(st.handle, 0, n + len(old))
    st.ids4 = K.kv_alloc_blocks(st.handle, 1, n4)
    view = buf[: ids.size * block // 2].view(-1, 2, Hkv, bs, d)
    view[:n], view[n:] = st.pages, old
    st.pages = view[:n]
    if len(old):
        K.kv_pack_blocks(st.handle, 0, 1, ids[n:], st.ids4)
        K.kv_free_blocks(st.handle, 0, ids[n:])
    if c["op"] != "decode":
        st.src, st.dst = (ids[x.cpu().numpy()] for x in (st.src, st.dst))
        return
    ids, ids4 = (torch.from_numpy(x).cuda() for x in (ids, np.append(st.ids4, -1).astype(np.int32)))
    st.table = torch.where(st.table < 0, -1, ids[st.table.clamp(min=0).long()])
    st.table4 = ids4[torch.where(st.table4 < 0, n4, st.table4).long()]
    st.ws_bytes = K.kv_q4_workspace_bytes(st.handle, 1, c["seqs"], Hq, st.max_blocks)
    st.ws = torch.empty(max(256, st.ws_bytes), dtype=torch.uint8, device="cuda")


# -------------------------------------------------------------- the call ---
def run(st):
    c = st.case
    if own:
        K, h, (Hq, _) = st.K, st.handle, _heads(c)
        if c["op"] == "norm":
            K.kv_append_rotary_norm(h, 0, st.rotary, st.norm, st.q, st.q.stride(0), st.q_out, st.k, st.k.stride(0), st.v,
                                    st.v.stride(0), None, st.starts if c["q_hi"] > 1 else None, st.T, st.table, st.lens,
                                    st.max_blocks, c["seqs"], Hq)
            return {"q": st.q_out, "pool": st.pages}
        if c["op"] == "decode":
            K.paged_decode_attn_q4(h, 0, 1, st.q, st.k, st.v, st.out, st.table, st.lens, st.max_blocks, st.table4,
                                   st.lens4, st.max_blocks, c["seqs"], Hq, st.scale, st.ws, st.ws_bytes)
            return {"out": st.out, "pool": st.pages}
        if c["op"] == "pack":
            K.kv_pack_blocks(h, 0, 1, st.src, st.ids4)
        K.kv_unpack_blocks(h, 1, 0, st.ids4, st.dst)
        return {"pool": st.pages}
    if c["op"] == "norm":
        return _plain_norm(st)
    if c["op"] == "decode":
        _put(st, st.k, st.v, torch.arange(c["seqs"], device="cuda"), st.lens.long() - 1)
        return {"out": _plain_attention(st), "pool": st.pages}
    st.pages[st.dst] = _values(*(_quantise(st.pages[st.src]) if c["op"] == "pack" else
                                 (st.codes, st.scales, st.least))).to(torch.bfloat16)
    return {"pool": st.pages}


def _put(st, k, v, seq, pos):
    """Rows k, v of tokens at positions pos of sequences seq into their pages."""
    bs = st.case["block"]
    blk = st.table[seq, pos // bs].long()
    shape = (len(pos), st.pages.shape[2], st.pages.shape[4])
    st.pages[blk, 0, :, pos % bs] = k.reshape(shape)
    st.pages[blk, 1, :, pos % bs] = v.reshape(shape)


def _quantise(x):
    """Codes, scales and least values of rows x [..., d] in groups of 64 columns.
    The quotients in 64 bits: a tie's neighbours are a whole code apart."""
    x = x.float().unflatten(-1, (-1, GROUP))
    z = x.amin(-1, keepdim=True)
    s = ((x.amax(-1, keepdim=True) - z) / 15.0).to(torch.bfloat16).float()
    codes = torch.round((x - z).double() / torch.where(s > 0, s, 1.0).double())
    return torch.where(s > 0, codes, 0.0).to(torch.uint8), s, z


def _values(codes, s, z):
    """The values that codes stand for, in 32 bits."""
    return (codes.float() * s + z).flatten(-2)


def _plain_norm(st):
    c, (Hq, Hkv), d, r = st.case, _heads(st.case), st.case["head_dim"], st.case["rot"]
    t = torch.arange(st.T, device="cuda")
    seq = (t.view(-1, 1) >= st.starts[1:]).sum(1)
    pos = (st.lens[seq] - st.starts[seq + 1] + t).long()
    angle = pos.double().view(-1, 1) * torch.from_numpy(st.freqs).cuda()
    cos, sin = (f(angle).float().unsqueeze(1) for f in (torch.cos, torch.sin))

    def turned(x, heads, weight):
        x = x.reshape(-1, heads, d).float()
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + st.eps) * (weight.float() + c["offset"])
        a, b = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        y = x.clone()
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y.to(torch.bfloat16)

    _put(st, turned(st.k, Hkv, st.k_weight), st.v, seq, pos)
    return {"q": turned(st.q, Hq, st.q_weight), "pool": st.pages}


def _plain_attention(st):
    """Every sequence's context gathered side by side, padded to the longest."""
    c, (Hq, Hkv), d, bs = st.case, _heads(st.case), st.case["head_dim"], st.case["block"]
    S, G = c["seqs"], Hq // Hkv
    j = torch.arange(st.max_len, device="cuda")
    late = (j >= st.lens4.view(-1, 1)) & (j < st.lens.view(-1, 1))
    seq, pos = late.nonzero(as_tuple=True)
    blk = st.table[seq, pos // bs].long()
    early = (j < st.lens4.view(-1, 1)).nonzero(as_tuple=True)
    old = st.table4[early[0], early[1] // bs].long()

    def rows(kv):  # [S, Hkv, max_len, d]
        x = torch.zeros(S, st.max_len, Hkv, d, device="cuda")
        at = (old, kv, slice(None), early[1] % bs)
        x[early] = _values(st.codes[at], st.scales[at], st.least[at])
        x[seq, pos] = st.pages[blk, kv, :, pos % bs].float()
        return x.transpose(1, 2)

    s = st.q.float().view(S, Hkv, G, d) @ rows(0).transpose(2, 3) * st.scale
    s = s.masked_fill_((j >= st.lens.view(-1, 1)).view(S, 1, 1, -1), float("-inf"))
    e = torch.exp_(s.sub_(s.amax(-1, keepdim=True)))
    o = e @ rows(1) / e.sum(-1, keepdim=True)
    st.out.copy_(o.reshape(S, Hq, d))
    return st.out


# ------------------------------------------------------- 64-bit answers ---
def _exact_values(x):
    """What rows x [..., d] read back as after packing, from the definition."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for a in range(0, x.shape[-1], GROUP):
        part = x[..., a : a + GROUP].double()
        low, high = part.min(-1, keepdim=True).values, part.max(-1, keepdim=True).values
        step = ((high - low) / 15).bfloat16().double()
        code = torch.nan_to_num((part - low) / step).round()
        out[..., a : a + GROUP] = low + code * step
    return out


def exact(case, seed):
    st = prepare(case, seed)
    c, (Hq, Hkv), d, bs = st.case, _heads(case), case["head_dim"], case["block"]
    if c["op"] in ("pack", "unpack"):
        want, src = st.pages.double(), st.old if c["op"] == "unpack" else st.pages[st.src]
        for b in range(0, len(src), 500):
            want[st.dst[b : b + 500]] = _exact_values(src[b : b + 500])
        return {"pool": want}
    starts, lens = st.starts.tolist(), st.lens.tolist()
    if c["op"] == "norm":
        f, r = torch.from_numpy(st.freqs).cuda(), c["rot"]
        pool, q_out = st.pages.double(), torch.empty(st.T, Hq, d, device="cuda", dtype=torch.float64)
        for s, n in enumerate(lens):
            rows = slice(starts[s], starts[s + 1])
            pos = torch.arange(n - starts[s + 1] + starts[s], n, device="cuda")
            turn = torch.exp(1j * (pos.double().view(-1, 1, 1) * f))
            out = []
            for x, h, w in ((st.q[rows], Hq, st.q_weight), (st.k[rows], Hkv, st.k_weight)):
                x = x.reshape(-1, h, d).double()
                x = x * (w.double() + c["offset"]) * (x.square().sum(-1, keepdim=True) / d + st.eps) ** -0.5
                pairs = x[..., :r].reshape(-1, h, r // 2, 2) if c["interleaved"] else \
                    x[..., :r].reshape(-1, h, 2, r // 2).transpose(2, 3)
                y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
                y = y if c["interleaved"] else y.transpose(2, 3)
                out.append(torch.cat([y.reshape(-1, h, r), x[..., r:]], -1))
            q_out[rows] = out[0]
            blk = st.table[s, pos // bs].long()
            pool[blk, 0, :, pos % bs] = out[1]
            pool[blk, 1, :, pos % bs] = st.v[rows].reshape(-1, Hkv, d).double()
        return {"q": q_out, "pool": pool}
    pages, old = st.pages.double(), st.lens4.tolist()
    out = torch.empty(len(lens), Hq, d, device="cuda", dtype=torch.float64)
    for s, n in enumerate(lens):
        last = pages[st.table[s, (n - 1) // bs].long()]
        last[0, :, (n - 1) % bs], last[1, :, (n - 1) % bs] = st.k[s].double(), st.v[s].double()
        b = old[s] // bs
        kv = torch.cat([_exact_values(st.old[st.table4[s, :b].long()]), pages[st.table[s, b : -(-n // bs)].long()]])
        kv = kv.permute(1, 2, 0, 3, 4).reshape(2, Hkv, -1, d)[:, :, :n]
        w = torch.einsum("hgd,hjd->hgj", st.q[s].view(Hkv, -1, d).double(), kv[0]) * st.scale
        out[s] = torch.einsum("hgj,hjd->hgd", torch.softmax(w, -1), kv[1]).reshape(Hq, d)
    return {"out": out, "pool": pages}
