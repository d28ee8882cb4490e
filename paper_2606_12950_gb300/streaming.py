"""One attention layer of a server: WindowedLayer, whose chats outgrow their
window (rotary positions, a sliding window with sinks, forks, and a page cache
that gives back what the window has left behind), and PackedLayer, whose chats
keep their whole context (heads normed, the older pages in 4 bits).

PyTorch supplies device memory and the stream; every step of the path runs in
libkvpool's kernels: the rotary append, prompt and decode attention over the
window, the copies of forked and moved pages.
"""
from __future__ import annotations

import contextlib

import numpy as np
import torch

from . import kvpool as K
from .runner import DevicePool


def _as_stream(stream, device):
    """A torch stream of a torch stream, a raw handle or an object that has one."""
    if hasattr(stream, "wait_stream"):
        return stream
    handle = int(getattr(stream, "cuda_stream", stream))
    if handle in (0, 1):  # the null stream, by either name
        return torch.cuda.default_stream(device)
    return torch.cuda.ExternalStream(handle, device)


class WindowedLayer:
    """Slots of one layer over a pool of pages.

    n_pages blocks of bs tokens; Hq query and Hkv KV heads of d columns;
    max_seqs slots of at most max_tokens tokens; a query sees the last `window`
    tokens and the first `sinks` (window 0: all).  freqs: the rotated pairs'
    frequencies (kvpool.kv_rotary_freqs), radians a position.  pool: a pool of
    the caller's with this layout as its first (e.g. runner.VmmPool, which gives
    physical memory back) in place of one of n_pages.

    Streams.  A call's `stream` (None: torch's current one) runs its kernels and
    owns what it allocates.  It waits first for the current stream, where q, k and
    v were made, and for the stream of the layer's call before.  The result is
    ready on `stream`: work elsewhere that reads it has to wait for that.  Where
    layers share a pool, calls on different streams are the caller's to order.
    """

    def __init__(self, n_pages: int, Hq: int, Hkv: int, d: int, bs: int, max_seqs: int, max_tokens: int, window: int,
                 sinks: int, freqs, interleaved: bool = False, magnitude: float = 1.0, scale: float | None = None, pool=None):
        self.Hq, self.Hkv, self.d, self.bs, self.S = Hq, Hkv, d, bs, max_seqs
        self.window, self.sinks = window, sinks
        self.scale = d ** -0.5 if scale is None else scale
        self.own = pool is None
        self.pool = DevicePool(n_pages, 2 * Hkv * bs * d * 2, bs, [(Hkv, d)]) if pool is None else pool
        dev = self.pool.device
        self.tab = K.SeqTab(self.pool.handle, 0, max_seqs, -(-max_tokens // bs))
        self.table = torch.empty((max_seqs, self.tab.max_blocks), dtype=torch.int32, device=dev)
        self.lens = torch.empty(max_seqs, dtype=torch.int32, device=dev)
        steps = torch.from_numpy(K.kv_rotary_steps(freqs).view(np.int64)).to(dev)
        self.rotary = K.Rotary(2 * len(freqs), steps, interleaved=interleaved, magnitude=magnitude)
        n = K.kv_workspace_bytes(self.pool.handle, 0, max_seqs, Hq, self.tab.max_blocks)
        self.ws = torch.empty(max(256, n), dtype=torch.uint8, device=dev)
        self.device = self.table.device  # (with its index)
        self._leave(torch.cuda.current_stream(self.device))

    def _leave(self, st) -> None:
        """Notes the last call's stream and what stands for its work: the stream,
        or an event where it is not torch's own (those end never) and may be gone
        by the next call.  (An event between two calls ends their overlap.)"""
        self.last = self.done = st
        self.handle, self.again = st.cuda_stream, contextlib.nullcontext(st)
        if st.cuda_stream and st.stream_id == st.cuda_stream:
            self.handle, self.done = -1, st.record_event()

    def _on(self, stream, *rows):
        """A call's stream, as a context that has it current and behind all that the
        call needs; `rows` are the caller's tensors."""
        # as most calls are (the handle alone: current_stream and a generator cost a
        # step of four slots 9 us of 41)
        if stream is None and torch._C._cuda_getCurrentRawStream(self.device.index) == self.handle:
            return self.again
        here = torch.cuda.current_stream(self.device)
        return self._go_to(here if stream is None else _as_stream(stream, self.device), here, rows)

    @contextlib.contextmanager
    def _go_to(self, st, here, rows):
        if st.cuda_stream != self.handle:  # (a stream that is not torch's may be a new one by an old handle)
            if self.done is self.last:
                st.wait_stream(self.last)
            else:
                st.wait_event(self.done)
            # (what torch's allocator has from another stream, it takes back after this one)
            for x in self._kept():
                x.record_stream(st)
        try:
            if st.cuda_stream == here.cuda_stream:
                yield st
            else:
                st.wait_stream(here)
                for x in rows:
                    x.record_stream(st)
                with torch.cuda.stream(st):
                    yield st
        finally:
            self._leave(st)

    def _kept(self) -> tuple:
        """The layer's own device tensors."""
        return self.table, self.lens, self.ws, self.rotary.steps

    def _workspace(self, n: int) -> torch.Tensor:
        if n > self.ws.numel():
            self.ws = torch.empty(n, dtype=torch.uint8, device=self.ws.device)
        return self.ws

    def _check_rows(self, T: int, q, k, v) -> None:
        """ValueError unless q, k and v are T rows each as the kernels read them
        (bf16 on the pool's device, a row's heads packed, rows 16 bytes apart or a
        multiple, from such an address; a row may hold more columns than are read)."""
        for name, x, heads in (("q", q, self.Hq), ("k", k, self.Hkv), ("v", v, self.Hkv)):
            shape, stride, row = x.shape, x.stride(), heads * self.d
            if len(shape) == 2 and stride[1] == 1:
                width = shape[1]  # columns of a row that follow one another
            else:
                width = 1
                for i in range(len(shape) - 1, 0, -1):
                    if shape[i] != 1 and stride[i] != width:
                        width = 0
                        break
                    width *= shape[i]
            if x.dtype is not torch.bfloat16 or x.device != self.device:
                raise ValueError(f"{name} must be bfloat16 on {self.device}, not {x.dtype} on {x.device}")
            if len(shape) < 2 or shape[0] != T or width < row:
                raise ValueError(f"{name} must hold {T} rows of {row} packed columns, not {tuple(shape)} with strides "
                                 f"{stride}")
            if x.data_ptr() % 16 or stride[0] % 8 or stride[0] < row:
                raise ValueError(f"{name}'s rows must lie apart, each at a multiple of 16 bytes")

    def _append(self, q, k, v, starts, T, stream):
        """q rotated into a new tensor; k rotated, k and v written to the pages."""
        q_out = torch.empty((T, self.Hq, self.d), dtype=torch.bfloat16, device=q.device)
        K.kv_append_rotary(self.pool.handle, 0, self.rotary, q, q.stride(0), q_out, k, k.stride(0), v, v.stride(0),
                           None, starts, T, self.table, self.lens, self.tab.max_blocks, self.S, self.Hq, stream)
        return q_out

    def prompt(self, counts, q, k, v, stream=None) -> torch.Tensor:
        """Append counts[s] new tokens to each slot s and attend: q, k, v hold
        their rows, slot after slot ([T, heads * d] bf16, any row stride).
        Returns [T, Hq, d].  ValueError where the rows do not fit (nothing has
        changed then); KVError (KV_ERR_OUT_OF_BLOCKS) where the pool cannot
        hold a slot's tokens; slots before it keep their reservation."""
        counts = np.asarray(counts, dtype=np.int64)
        lens, T = self.tab.lens(), int(counts.sum())
        if counts.shape != (self.S,) or counts.min() < 0 or q.shape[0] != T:
            raise ValueError("counts must have a number for each slot, and q a row for each new token")
        if T:
            self._check_rows(T, q, k, v)
        for s in np.nonzero(counts)[0]:
            self.tab.reserve(int(s), int(lens[s] + counts[s]))
        for s in np.nonzero(counts)[0]:
            self.tab.set_len(int(s), int(lens[s] + counts[s]))
        if T == 0:
            return torch.empty((0, self.Hq, self.d), dtype=torch.bfloat16, device=q.device)
        with self._on(stream, q, k, v) as st:
            out = torch.empty((T, self.Hq, self.d), dtype=torch.bfloat16, device=q.device)
            starts = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(q.device)
            self.tab.sync(self.table, self.lens, st)
            x = self._append(q, k, v, starts, T, st)
            n = K.kv_prompt_workspace_bytes(self.pool.handle, 0, self.S, self.Hq, T, int(counts.max()),
                                            self.tab.max_blocks, self.window, self.sinks)
            K.paged_prompt_attn(self.pool.handle, 0, x, out, starts, T, int(counts.max()), self.table, self.lens,
                                self.tab.max_blocks, self.S, self.Hq, self.scale, self.window, self.sinks,
                                self._workspace(n), n, st)
        self._evict(np.nonzero(counts)[0])
        return self._given(out, stream)

    def step(self, q, k, v, stream=None) -> torch.Tensor:
        """One decode step: a new token for every slot that holds a context (rows
        of the others are passed over).  q, k, v: a row per slot.  Returns
        [max_seqs, Hq, d], zeros for empty slots.  ValueError where the rows do
        not fit (nothing has changed then)."""
        self._check_rows(self.S, q, k, v)
        self.tab.advance()
        with self._on(stream, q, k, v) as st:
            self.tab.sync(self.table, self.lens, st)
            x = self._append(q, k, v, None, self.S, st)
            out = torch.empty_like(x)
            K.paged_decode_attn_window(self.pool.handle, 0, x, None, None, out, self.table, self.lens,
                                       self.tab.max_blocks, self.S, self.Hq, self.scale, self.window, self.sinks, 0,
                                       self.ws, self.ws.numel(), st)
        self._evict(np.nonzero(self.tab.lens())[0])
        return self._given(out, stream)

    def _given(self, out, stream) -> torch.Tensor:
        """The result, which the caller may read where it called."""
        if stream is not None:
            out.record_stream(torch.cuda.current_stream(out.device))
        return out

    def _evict(self, slots) -> None:
        if self.window:
            for s in slots:
                self.tab.evict(int(s), self.window, self.sinks)

    def fork(self, src: int, dsts, stream=None) -> None:
        with self._on(stream) as st:
            self.tab.fork(src, dsts, st)

    def release(self, s: int) -> None:
        self.tab.release(s)

    def compact(self, stream=None) -> int:
        """Pages moved together and whole free chunks given back; returns the
        number of pages moved.  (The next prompt or step sends the changed
        entries.)"""
        with self._on(stream) as st:
            moved = K.kv_pool_compact(self.pool.handle, stream=st)
        K.kv_pool_trim(self.pool.handle)
        return moved

    def pages_used(self) -> int:
        return K.kv_pool_stats(self.pool.handle)["blocks_used"][0]

    def close(self) -> None:
        torch.cuda.synchronize()
        self.tab.close()
        if self.own:
            self.pool.close()


class PackedLayer(WindowedLayer):
    """Slots of one layer that see their whole context, of which the older pages
    are held in 4 bits: every full page but those that the last `keep` tokens
    reach (at least 1) is packed at the end of the call that filled it.

    n_pages: the pool's size in bf16 pages, each of which has room for three
    packed ones (pool: a pool of the caller's whose layouts are (Hkv, d) and (Hkv,
    d | KV_Q4)).  norm: the heads' norms (kvpool.HeadNorm), or None.  The rest, the
    streams too, is as WindowedLayer says.  Where the pool has no page left for
    packing, a slot's pages stay in bf16 until a later call finds one.  A prompt on a chat
    with packed pages reads them through bf16 copies, which it needs pages for
    while it runs.
    """

    def __init__(self, n_pages: int, Hq: int, Hkv: int, d: int, bs: int, max_seqs: int, max_tokens: int, keep: int, freqs,
                 norm=None, interleaved: bool = False, magnitude: float = 1.0, scale: float | None = None, pool=None):
        if keep < 1:
            raise ValueError("keep must be at least 1")
        own = pool is None
        if own:
            pool = DevicePool(32 * n_pages, Hkv * bs * d // 8, bs, [(Hkv, d), (Hkv, d | K.KV_Q4)])
        self.norm, self.keep = norm, keep
        self.tab4 = K.SeqTab(pool.handle, 1, max_seqs, -(-max_tokens // bs))
        self.table4 = torch.empty((max_seqs, self.tab4.max_blocks), dtype=torch.int32, device=pool.device)
        self.lens4 = torch.empty(max_seqs, dtype=torch.int32, device=pool.device)
        super().__init__(n_pages, Hq, Hkv, d, bs, max_seqs, max_tokens, 0, 0, freqs, interleaved, magnitude, scale, pool)
        self.own = own
        n = K.kv_q4_workspace_bytes(pool.handle, 1, max_seqs, Hq, self.tab.max_blocks)
        self._workspace(n)

    def _kept(self) -> tuple:
        weights = () if self.norm is None else tuple(w for w in self.norm.weights if w is not None)
        return super()._kept() + (self.table4, self.lens4) + weights

    def _append(self, q, k, v, starts, T, stream):
        if self.norm is None:
            return super()._append(q, k, v, starts, T, stream)
        q_out = torch.empty((T, self.Hq, self.d), dtype=torch.bfloat16, device=q.device)
        K.kv_append_rotary_norm(self.pool.handle, 0, self.rotary, self.norm, q, q.stride(0), q_out, k, k.stride(0), v,
                                v.stride(0), None, starts, T, self.table, self.lens, self.tab.max_blocks, self.S, self.Hq,
                                stream)
        return q_out

    def _room(self, call):
        """call(), once more with the pages that the other kind has free where there
        are none (a pool keeps those until kv_pool_trim)."""
        try:
            return call()
        except K.KVError as e:
            if e.code != K.KV_ERR_OUT_OF_BLOCKS:
                raise
        K.kv_pool_trim(self.pool.handle)
        return call()

    def _pack(self, slots, st) -> None:
        try:
            self._room(lambda: self.tab.pack(self.tab4, slots, self.keep, st))
            return
        except K.KVError as e:
            if e.code != K.KV_ERR_OUT_OF_BLOCKS:
                raise
        # a few pages at a time, oldest first: those that become free make room for the next
        lens, done = self.tab.lens(), self.tab4.lens()
        for s in slots:
            want, have = max(0, int(lens[s]) - self.keep) // self.bs, int(done[s]) // self.bs
            while have < want:
                K.kv_pool_trim(self.pool.handle)
                st4 = K.kv_pool_stats(self.pool.handle)
                n = min(want - have, st4["blocks_capacity"][1] - st4["blocks_used"][1])
                # (a VMM pool's capacity counts what its limit or budget may not let be mapped)
                while n and not self._packs(s, int(lens[s]) - (have + n) * self.bs, st):
                    n //= 2
                if n == 0:
                    return  # they stay as they are until there is room
                have += n

    def _packs(self, s: int, keep: int, st) -> bool:
        """Packs slot s but for its last `keep` tokens; False where there is no room."""
        try:
            self.tab.pack(self.tab4, [s], keep, st)
        except K.KVError as e:
            if e.code != K.KV_ERR_OUT_OF_BLOCKS:
                raise
            return False
        return True

    def prompt(self, counts, q, k, v, stream=None) -> torch.Tensor:
        """As WindowedLayer.prompt; KVError (KV_ERR_OUT_OF_BLOCKS) also where the
        pool has no pages for copies of packed ones (nothing has changed then)."""
        counts = np.asarray(counts, dtype=np.int64)
        lens, T = self.tab.lens(), int(counts.sum())
        if counts.shape != (self.S,) or counts.min() < 0 or q.shape[0] != T:
            raise ValueError("counts must have a number for each slot, and q a row for each new token")
        if T == 0:
            return torch.empty((0, self.Hq, self.d), dtype=torch.bfloat16, device=q.device)
        self._check_rows(T, q, k, v)
        slots = np.nonzero(counts)[0]
        table4, lens4 = self.tab4.host()
        packed = [(s, int(lens4[s]) // self.bs) for s in slots if lens4[s]]
        # (first: without them nothing is reserved)
        copies = self._room(lambda: K.kv_alloc_blocks(self.pool.handle, 0, sum(n for _, n in packed)))
        try:
            for s in slots:
                self._room(lambda: self.tab.reserve(int(s), int(lens[s] + counts[s])))
            for s in slots:
                self.tab.set_len(int(s), int(lens[s] + counts[s]))
            with self._on(stream, q, k, v) as st:
                out = torch.empty((T, self.Hq, self.d), dtype=torch.bfloat16, device=q.device)
                starts = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(q.device)
                self.tab.sync(self.table, self.lens, st)
                table, ctx = self.table, self.lens
                if packed:
                    K.kv_unpack_blocks(self.pool.handle, 1, 0, np.concatenate([table4[s, :n] for s, n in packed]), copies, st)
                    whole, at = self.tab.host()[0], 0
                    for s, n in packed:
                        whole[s, :n] = copies[at : at + n]
                        at += n
                    # (the other slots have no rows here, and what they see is not asked for)
                    ctx = torch.from_numpy(np.where(counts > 0, lens + counts, 0).astype(np.int32)).to(q.device)
                    table = torch.from_numpy(whole).to(q.device)
                x = self._append(q, k, v, starts, T, st)
                n = K.kv_prompt_workspace_bytes(self.pool.handle, 0, self.S, self.Hq, T, int(counts.max()),
                                                self.tab.max_blocks, 0, 0)
                K.paged_prompt_attn(self.pool.handle, 0, x, out, starts, T, int(counts.max()), table, ctx,
                                    self.tab.max_blocks, self.S, self.Hq, self.scale, 0, 0, self._workspace(n), n, st)
                self._pack(slots, st)
        finally:
            if copies.size:
                K.kv_free_blocks(self.pool.handle, 0, copies)
        return self._given(out, stream)

    def step(self, q, k, v, stream=None) -> torch.Tensor:
        """As WindowedLayer.step."""
        self._check_rows(self.S, q, k, v)
        self._room(self.tab.advance)
        with self._on(stream, q, k, v) as st:
            self.tab.sync(self.table, self.lens, st)
            self.tab4.sync(self.table4, self.lens4, st)
            x = self._append(q, k, v, None, self.S, st)
            out = torch.empty_like(x)
            K.paged_decode_attn_q4(self.pool.handle, 0, 1, x, None, None, out, self.table, self.lens, self.tab.max_blocks,
                                   self.table4, self.lens4, self.tab4.max_blocks, self.S, self.Hq, self.scale, self.ws,
                                   self.ws.numel(), st)
            self._pack(np.nonzero(self.tab.lens())[0], st)
        return self._given(out, stream)

    def fork(self, src: int, dsts, stream=None) -> None:
        dsts = np.asarray(dsts, dtype=np.int32)
        self._room(lambda: super(PackedLayer, self).fork(src, dsts, stream))
        try:
            self.tab4.fork(src, dsts)  # whole pages, by reference
        except K.KVError:
            for s in dsts:
                self.tab.release(int(s))
            raise

    def release(self, s: int) -> None:
        self.tab.release(s)
        self.tab4.release(s)

    def packed_used(self) -> int:
        """Pages held in 4 bits (pages_used: in bf16)."""
        return K.kv_pool_stats(self.pool.handle)["blocks_used"][1]

    def close(self) -> None:
        torch.cuda.synchronize()
        self.tab4.close()
        super().close()
