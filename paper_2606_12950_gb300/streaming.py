"""One attention layer of a server whose chats outgrow their window: rotary
positions, a sliding window with sinks, forks, and a page cache that gives back
what the window has left behind.

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
            for x in (self.table, self.lens, self.ws, self.rotary.steps):
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
