"""The operators of a layer with rotary positions, sliding-window attention and
a managed page cache, as measurable cases.

One pass is one call on one layer's paged bf16 cache ([K|V][Hkv][block][d] per
block, reached through a block table):

  rotary   the new tokens' q and k rotated to their positions, k and v written
           into the cache: one token a sequence, or ragged prompt chunks
  decode   one query a sequence over the last `window` tokens and the first
           `sinks` ones, the step's new K/V row appended in the same call
  prompt   the queries of ragged prompt chunks, causally, with the same mask
           (window 0: over the whole context)
  copy     pages, or the first tokens of pages, copied to other pages: forked
           sequences' partial last pages, pages moved together

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


def _case(name, op, seqs, heads, *, head_dim=128, block=16, ctx="uniform", lo=0, hi=0, q_lo=1, q_hi=1, window=0,
          sinks=0, evicted=False, rot=0, interleaved=False, stretch=1.0, tok_lo=0):
    """heads: query x KV heads.  ctx, lo, hi: cached tokens before the call.
    q_lo, q_hi: the call's new tokens a sequence.  evicted: the table holds no
    pages outside the window and the sinks.  rot: rotated columns of a head;
    stretch: the context's extension over the trained 8192 tokens.  copy: seqs
    pages of block tokens, of which tok_lo .. block are copied."""
    c = {"op": op, "seqs": seqs, "heads": heads, "head_dim": head_dim, "block": block, "ctx": ctx, "lo": lo, "hi": hi,
         "q_lo": q_lo, "q_hi": q_hi, "window": window, "sinks": sinks, "evicted": evicted, "rot": rot,
         "interleaved": interleaved, "stretch": stretch, "tok_lo": tok_lo}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest model of the tests, a step of four short chats
        _case("rotary_tiny_step", "rotary", 4, "4x2", head_dim=64, lo=17, hi=255, rot=64),
        # an ordinary decode batch's step: rows of one fused projection
        _case("rotary_step", "rotary", 64, "32x8", ctx="lognormal", lo=1024, hi=16384, rot=128),
        # admitted prompts late in long contexts, half of each head rotated in
        # adjacent pairs, frequencies stretched eightfold
        _case("rotary_prompts", "rotary", 24, "40x8", lo=5, hi=60000, q_lo=3, q_hi=1333, rot=64, interleaved=True,
              stretch=8.0),
        # one user's long chat: only the window's and the sinks' pages are held
        _case("decode_long_chat", "decode", 1, "32x8", lo=50000, hi=50000, window=4096, sinks=4, evicted=True),
        # an ordinary batch, some chats still shorter than the window
        _case("decode_batch", "decode", 64, "32x8", ctx="lognormal", lo=1500, hi=16384, window=1024, sinks=4,
              evicted=True),
        # a large batch of long contexts, pages of 32 tokens, nothing freed yet
        _case("decode_many", "decode", 250, "32x8", block=32, ctx="pareto", lo=300, hi=12000, window=2048, sinks=20),
        # a first short prompt of the smallest model
        _case("prompt_tiny", "prompt", 1, "4x2", head_dim=64, q_lo=33, q_hi=33),
        # ragged chunks beside single tokens, on chats of all lengths
        _case("prompt_chunks", "prompt", 9, "32x8", lo=0, hi=7000, q_lo=1, q_hi=700, window=1024, sinks=4,
              evicted=True),
        # a long document in one call
        _case("prompt_document", "prompt", 1, "32x8", q_lo=16384, q_hi=16384, window=4096, sinks=4),
        # full causal prompts of a small model without grouped heads
        _case("prompt_causal", "prompt", 5, "16x16", head_dim=64, block=32, lo=0, hi=600, q_lo=700, q_hi=2500),
        # agents forked from running chats: the partial last pages
        _case("copy_fork", "copy", 48, "32x8", tok_lo=1),
        # pages moved together so that memory can be given back
        _case("copy_compact", "copy", 4000, "32x8", tok_lo=16),
    ]


# no drawn case costs more than the largest listed one of its kind
_MOST = {"rotary": 4.2e8, "decode": 1.9e9, "prompt": 1.1e12, "copy": 5.2e8}


def draw(rng):
    """A case of the same ranges."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotary", "decode", "decode", "prompt", "prompt", "copy"])
    head_dim, block = rng.choice([64, 128, 128]), rng.choice([16, 16, 32, 64])
    kv = rng.choice([1, 2, 4, 8, 8, 16])
    heads = "%dx%d" % (kv * rng.choice([1, 2, 4, 4, 5, 8]), kv)
    ctx, window, sinks = rng.choice(["uniform", "lognormal", "pareto"]), log_int(40, 6000), rng.randrange(0, 40)
    common = dict(head_dim=head_dim, block=block, ctx=ctx)
    if op == "rotary":
        q_hi = rng.choice([1, log_int(2, 4000)])
        c = _case("", op, log_int(1, 400), heads, lo=rng.randrange(0, 400), hi=log_int(400, 100000), q_lo=1, q_hi=q_hi,
                  rot=rng.choice([16, 32, 64, head_dim, head_dim]), interleaved=rng.random() < 0.5,
                  stretch=rng.choice([1.0, 1.0, 4.0, 16.0]), **common)
    elif op == "decode":
        c = _case("", op, log_int(1, 400), heads, lo=rng.randrange(0, 700), hi=log_int(700, 60000), window=window,
                  sinks=sinks, evicted=rng.random() < 0.7, **common)
    elif op == "prompt":
        if rng.random() < 0.3:
            window = sinks = 0
        q_hi = log_int(2, 12000)
        c = _case("", op, log_int(1, 24), heads, lo=rng.randrange(0, 300), hi=log_int(300, 16000), q_lo=rng.randrange(
            0, q_hi), q_hi=q_hi, window=window, sinks=sinks, evicted=window > 0 and rng.random() < 0.7, **common)
    else:
        c = _case("", op, log_int(8, 6000), heads, head_dim=head_dim, block=block, tok_lo=rng.randrange(1, block + 1))
    while _cost(c) > _MOST[op] or _footprint(c) > 3.0e10:
        if c["seqs"] > 1:
            c["seqs"] = c["seqs"] * 3 // 4
        else:
            c["q_hi"] = max(1, c["q_hi"] * 3 // 4)
            c["q_lo"] = min(c["q_lo"], c["q_hi"])
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


def _visible(p, window, sinks):
    """Tokens that a query at position p sees."""
    n = p + 1
    return n if not window else np.minimum(n, window) + np.minimum(sinks, np.maximum(0, n - window))


def _page_tokens(c):
    """Copied tokens of each page."""
    return c["tok_lo"] + np.arange(c["seqs"]) * (c["block"] - c["tok_lo"] + 1) // c["seqs"]


def work(c):
    Hq, Hkv = _heads(c)
    row = 2 * c["head_dim"]  # bytes of a head's row
    if c["op"] == "copy":
        return {"bytes": int(_page_tokens(c).sum()) * 2 * Hkv * row * 2, "flops": 0}
    nq, n = _sizes(c)
    T = int(nq.sum())
    if c["op"] == "rotary":
        return {"bytes": T * 2 * (Hq + 2 * Hkv) * row, "flops": T * (Hq + Hkv) * c["rot"] * 3}
    window, sinks = c["window"], c["sinks"]
    pairs = sum(int(_visible(np.arange(b - a, b), window, sinks).sum()) for a, b in zip(nq, n))
    first = np.maximum(0, n - nq - window + 1) if window else np.zeros_like(n)
    keys = int(np.where(nq > 0, n - first + np.minimum(sinks, first), 0).sum())
    byts = keys * 2 * Hkv * row + T * 2 * Hq * row
    if c["op"] == "decode":
        byts += T * 2 * Hkv * row
    return {"bytes": byts, "flops": pairs * Hq * c["head_dim"] * 4}


def _cost(c):
    w = work(c)
    return w["flops"] if c["op"] == "prompt" else w["bytes"]


def _query_block(c):
    return 1 if c["op"] == "decode" else min(64, max(1, c["q_hi"]))


def _footprint(c):
    """About what the plain form holds at its largest."""
    Hq, Hkv = _heads(c)
    nq, n = _sizes(c)
    if c["op"] in ("rotary", "copy"):
        return int(n.max()) * 4 if c["op"] == "copy" else int(nq.sum()) * Hq * c["head_dim"] * 32
    bq = _query_block(c)
    rows = c["seqs"] * -(-max(1, int(nq.max())) // bq)
    cols = min(c["window"] or 1 << 40, int(n.max())) + bq + c["sinks"]
    return rows * cols * (Hkv * c["head_dim"] * 16 + Hq * bq * 12)


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

    if c["op"] == "copy":
        n_pages = 2 * S + S // 9 + 8
        ids = rng.permutation(n_pages).astype(np.int32)
        st.src, st.dst = ids[:S].copy(), ids[S : 2 * S].copy()
        st.tokens = rng.permutation(_page_tokens(c)).astype(np.int32)
    else:
        nq, n = _sizes(c)
        order = rng.permutation(S)
        nq, n = nq[order], n[order]
        st.max_q, st.max_len, st.T = int(nq.max()), int(n.max()), int(nq.sum())
        st.max_blocks = max(1, -(-st.max_len // bs))
        blocks = -(-n // bs)
        at = np.arange(st.max_blocks)
        held = at < blocks[:, None]
        if c["evicted"]:  # neither in the first query's window nor among the sinks
            first = np.maximum(0, n - nq - c["window"] + 1)
            held &= (at < -(-c["sinks"] // bs)) | (at >= (first // bs)[:, None])
        if c["op"] == "rotary":  # the pages that the call writes
            held &= at >= ((n - nq) // bs)[:, None]
        n_held = int(held.sum())
        n_pages = n_held + n_held // 9 + 8
        table = np.full(held.shape, -1, dtype=np.int32)
        table[held] = rng.permutation(n_pages)[:n_held]
        st.table = torch.from_numpy(table).cuda()
        st.lens = torch.from_numpy(n.astype(np.int32)).cuda()
        st.starts = torch.from_numpy(np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)).cuda()
        st.ragged = c["op"] == "prompt" or c["q_hi"] > 1
        st.scale = d ** -0.5
    st.pages = normal(n_pages, 2, Hkv, bs, d)
    if c["op"] == "rotary":
        qkv = normal(st.T, (Hq + 2 * Hkv) * d)  # rows of one fused projection
        st.q, st.k, st.v = qkv[:, : Hq * d], qkv[:, Hq * d : (Hq + Hkv) * d], qkv[:, (Hq + Hkv) * d :]
        st.q_out = torch.empty(st.T, Hq, d, device="cuda", dtype=torch.bfloat16)
        st.freqs = _freqs(c)
        st.gain = 0.1 * math.log(c["stretch"]) + 1.0
    elif c["op"] != "copy":
        st.q = normal(st.T, Hq, d)
        st.out = torch.empty(st.T, Hq, d, device="cuda", dtype=torch.bfloat16)
        if c["op"] == "decode":
            st.k, st.v = normal(st.T, Hkv, d), normal(st.T, Hkv, d)
    if own:  # the pool's handle and what its calls keep: no input is touched
        _open(st, n_pages)
    return st


def _freqs(c):
    """Radians a position of each rotated pair, in 64 bits: base 500000; where
    the context is stretched, frequencies with fewer than one turn in 8192
    tokens divided by it, those with over 32 kept, between them in proportion."""
    f = 500000.0 ** (-2.0 * np.arange(c["rot"] // 2) / c["rot"])
    keep = np.clip((8192 * f / (2 * math.pi) - 1) / (32 - 1), 0, 1)
    return f * keep + f / c["stretch"] * (1 - keep) if c["stretch"] != 1 else f


def _open(st, n_pages):
    from paper_2606_12950_gb300 import kvpool as K

    st.K, c = K, st.case
    Hq, Hkv = _heads(c)
    st.err = torch.zeros(1, dtype=torch.int32, device="cuda")
    st.handle = K.kv_pool_create(st.pages, st.pages.numel() * 2, c["block"], [(Hkv, c["head_dim"])], st.err)
    K.kv_alloc_blocks(st.handle, 0, n_pages)
    if c["op"] == "rotary":
        st.steps = torch.from_numpy(K.kv_rotary_steps(st.freqs).view(np.int64)).cuda()
        st.rotary = K.Rotary(c["rot"], st.steps, interleaved=c["interleaved"], magnitude=st.gain)
    elif c["op"] == "decode":
        st.ws_bytes = K.kv_workspace_bytes(st.handle, 0, c["seqs"], Hq, st.max_blocks, 0)
    elif c["op"] == "prompt":
        st.ws_bytes = K.kv_prompt_workspace_bytes(st.handle, 0, c["seqs"], Hq, st.T, st.max_q, st.max_blocks,
                                                  c["window"], c["sinks"])
    if c["op"] in ("decode", "prompt"):
        st.ws = torch.empty(max(256, st.ws_bytes), dtype=torch.uint8, device="cuda")


# -------------------------------------------------------------- the call ---
def run(st):
    c = st.case
    if own:
        K, h, (Hq, _) = st.K, st.handle, _heads(c)
        if c["op"] == "rotary":
            K.kv_append_rotary(h, 0, st.rotary, st.q, st.q.stride(0), st.q_out, st.k, st.k.stride(0), st.v,
                               st.v.stride(0), None, st.starts if st.ragged else None, st.T, st.table, st.lens,
                               st.max_blocks, c["seqs"], Hq)
            return {"q": st.q_out, "pool": st.pages}
        if c["op"] == "decode":
            K.paged_decode_attn_window(h, 0, st.q, st.k, st.v, st.out, st.table, st.lens, st.max_blocks, c["seqs"], Hq,
                                       st.scale, c["window"], c["sinks"], 0, st.ws, st.ws_bytes)
            return {"out": st.out, "pool": st.pages}
        if c["op"] == "prompt":
            K.paged_prompt_attn(h, 0, st.q, st.out, st.starts, st.T, st.max_q, st.table, st.lens, st.max_blocks,
                                c["seqs"], Hq, st.scale, c["window"], c["sinks"], st.ws, st.ws_bytes)
            return {"out": st.out}
        K.kv_copy_blocks(h, 0, st.src, st.dst, st.tokens)
        return {"pool": st.pages}
    if c["op"] == "rotary":
        return _plain_rotary(st)
    if c["op"] == "decode":
        _put(st, st.k, st.v, torch.arange(c["seqs"], device="cuda"), st.lens.long() - 1)
        return {"out": _plain_attention(st), "pool": st.pages}
    if c["op"] == "prompt":
        return {"out": _plain_attention(st)}
    src, dst, tokens = (torch.from_numpy(a).cuda().long() for a in (st.src, st.dst, st.tokens))
    inside = torch.arange(c["block"], device="cuda") < tokens.view(-1, 1)
    inside = inside.view(-1, 1, 1, c["block"], 1)
    st.pages[dst] = torch.where(inside, st.pages[src], st.pages[dst])
    return {"pool": st.pages}


def _put(st, k, v, seq, pos):
    """Rows k, v of tokens at positions pos of sequences seq into their pages."""
    bs = st.case["block"]
    blk = st.table[seq, pos // bs].long()
    shape = (len(pos), st.pages.shape[2], st.pages.shape[4])
    st.pages[blk, 0, :, pos % bs] = k.reshape(shape)
    st.pages[blk, 1, :, pos % bs] = v.reshape(shape)


def _plain_rotary(st):
    c, (Hq, Hkv), d, r = st.case, _heads(st.case), st.case["head_dim"], st.case["rot"]
    t = torch.arange(st.T, device="cuda")
    seq = (t.view(-1, 1) >= st.starts[1:]).sum(1)
    pos = (st.lens[seq] - st.starts[seq + 1] + t).long()
    angle = pos.float().view(-1, 1) * torch.from_numpy(st.freqs).cuda().float()
    cos, sin = (f(angle).unsqueeze(1) * st.gain for f in (torch.cos, torch.sin))

    def rotated(x, heads):
        x = x.reshape(-1, heads, d).float()
        a, b = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        y = x.clone()
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y.to(torch.bfloat16)

    _put(st, rotated(st.k, Hkv), st.v, seq, pos)
    return {"q": rotated(st.q, Hq), "pool": st.pages}


def _plain_attention(st):
    """Queries in blocks of consecutive ones, each block with its band of keys
    and the sinks before it."""
    c, (Hq, Hkv), d, bs = st.case, _heads(st.case), st.case["head_dim"], st.case["block"]
    S, G, B = c["seqs"], Hq // Hkv, _query_block(c)
    W = min(c["window"] or st.max_len, st.max_len)
    nb = -(-max(1, st.max_q) // B)
    one = torch.arange
    starts, lens = st.starts.long(), st.lens.long()
    i = one(nb * B, device="cuda").view(1, nb, B)
    rows = starts[:-1].view(S, 1, 1) + i
    real = rows < starts[1:].view(S, 1, 1)
    p = (lens - starts[1:] + starts[:-1]).view(S, 1, 1) + i  # positions of the queries
    j = torch.cat([one(c["sinks"], device="cuda").expand(S, nb, -1),
                   p[:, :, :1] - W + 1 + one(W + B - 1, device="cuda")], 2).unsqueeze(2)
    sink = (one(j.shape[3], device="cuda") < c["sinks"]).view(1, 1, 1, -1)
    seen = torch.where(sink, j <= p.unsqueeze(3) - W, (j >= 0) & (j <= p.unsqueeze(3)) & (j > p.unsqueeze(3) - W))
    j = j.squeeze(2).clamp(0, st.max_blocks * bs - 1)
    blk = st.table[one(S, device="cuda").view(S, 1, 1), j // bs].long().clamp(min=0)
    k, v = (st.pages[blk, kv, :, j % bs].float().transpose(2, 3) for kv in (0, 1))  # [S, nb, Hkv, keys, d]
    q = st.q[rows.clamp(max=st.T - 1)].float().view(S, nb, B, Hkv, G, d).permute(0, 1, 3, 4, 2, 5)
    s = (q.reshape(S, nb, Hkv, G * B, d) @ k.transpose(3, 4) * st.scale).view(S, nb, Hkv, G, B, -1)
    s = s.masked_fill_(~seen.view(S, nb, 1, 1, B, -1), float("-inf"))
    e = torch.exp_(s.sub_(s.amax(-1, keepdim=True).clamp(min=-3e38)))
    o = (e.view(S, nb, Hkv, G * B, -1) @ v).view(S, nb, Hkv, G, B, d) / e.sum(-1, keepdim=True)
    o = o.permute(0, 1, 4, 2, 3, 5).reshape(S, nb, B, Hq, d)
    st.out[rows[real]] = o[real].to(torch.bfloat16)
    return st.out


# ------------------------------------------------------- 64-bit answers ---
def exact(case, seed):
    st = prepare(case, seed)
    c, (Hq, Hkv), d, bs = st.case, _heads(case), case["head_dim"], case["block"]
    if c["op"] == "copy":
        want = st.pages.double()
        for a, b, n in zip(st.src.tolist(), st.dst.tolist(), st.tokens.tolist()):
            want[b, :, :, :n] = st.pages[a, :, :, :n].double()
        return {"pool": want}
    starts, lens = st.starts.tolist(), st.lens.tolist()
    if c["op"] == "rotary":
        f, r = torch.from_numpy(st.freqs).cuda(), c["rot"]
        pool, q_out = st.pages.double(), torch.empty(st.T, Hq, d, device="cuda", dtype=torch.float64)
        for s, n in enumerate(lens):
            rows = slice(starts[s], starts[s + 1])
            pos = torch.arange(n - starts[s + 1] + starts[s], n, device="cuda")
            turn = torch.exp(1j * (pos.double().view(-1, 1, 1) * f)) * st.gain
            out = []
            for x, h in ((st.q[rows], Hq), (st.k[rows], Hkv)):
                x = x.reshape(-1, h, d).double()
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
    pages = st.pages
    if c["op"] == "decode":
        for s, n in enumerate(lens):
            pages[st.table[s, (n - 1) // bs].long(), 0, :, (n - 1) % bs] = st.k[s]
            pages[st.table[s, (n - 1) // bs].long(), 1, :, (n - 1) % bs] = st.v[s]
    out = torch.empty(st.T, Hq, d, device="cuda", dtype=torch.float64)
    for s, n in enumerate(lens):
        for a in range(starts[s], starts[s + 1], 512):
            b = min(a + 512, starts[s + 1])
            p = torch.arange(n - starts[s + 1] + a, n - starts[s + 1] + b, device="cuda")
            lo = max(0, int(p[0]) - c["window"] + 1) if c["window"] else 0
            j = torch.cat([torch.arange(min(c["sinks"], lo), device="cuda"), torch.arange(lo, int(p[-1]) + 1, device="cuda")])
            kv = pages[st.table[s, j // bs].long(), :, :, j % bs].double()  # [keys, 2, Hkv, d]
            hidden = j > p.view(-1, 1)
            if c["window"]:
                hidden |= (j <= p.view(-1, 1) - c["window"]) & (j >= c["sinks"])
            w = torch.einsum("thgd,jhd->hgtj", st.q[a:b].view(-1, Hkv, Hq // Hkv, d).double(), kv[:, 0]) * st.scale
            w = torch.softmax(w.masked_fill(hidden, float("-inf")), -1)
            out[a:b] = torch.einsum("hgtj,jhd->thgd", w, kv[:, 1]).reshape(-1, Hq, d)
    return {"out": out, "pool": pages.double()} if c["op"] == "decode" else {"out": out}
