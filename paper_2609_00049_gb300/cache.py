"""Generating with an 8-bit key/value cache: sequences in pages, their new tokens'
rotary positions, keys and values appended, attention over what is cached.

    cache = Cache8(layers, n_pages, rows, max_tokens, n_kv=8, head_dim=128)
    step = cache.begin([5, 0, 1])                       # new tokens of each row's sequence
    for layer in range(layers):
        out = cache.attend(step, layer, q, k, v)        # tokens x heads x head_dim; q and k are turned in place
    cache.fork([0], [1])                                # row 1 goes on from row 0's sequence, sharing its pages
    cache.release([0])
    cache.compact()

A step's rows are the table's: row s has `counts[s]` new tokens (0: it waits), which
lie one row's after the other's in q, k and v.  `begin` takes the pages
(realq_pages_reserve), `attend` runs realq_rotary, realq_kv_append and
realq_kv_attention; the modules around it are the caller's
(realq_int8_product on the sweep's codes, for instance).  Everything is enqueued
on the current stream (or `stream`); nothing is read back but by `check`, which
raises RealqError where the pool had too few pages: the step's tokens then have
position -1, and appending them does nothing.  Buffers are allocated with torch;
no arithmetic happens here.
"""
from __future__ import annotations

import contextlib
from dataclasses import dataclass
from typing import Optional, Sequence, Union

import torch

from . import (REALQ_ERR_TIMEOUT, RealqError, kv_cache, kv_pages, realq_kv_append, realq_kv_attention, realq_kv_attention_workspace_size,
               realq_pages_compact, realq_pages_fork, realq_pages_release, realq_pages_reserve,
               realq_pages_workspace_size, realq_rotary, realq_rotary_frequencies, realq_workspace_status, workspace, _heads,
               _ints as _buffer, _stream)

Rows = Union[Sequence[int], torch.Tensor]
_HERE = contextlib.nullcontext()


@dataclass
class Step:
    """One step's tokens: where each row's begin, their positions, the most of a row."""
    starts: torch.Tensor      # rows + 1
    positions: torch.Tensor   # tokens
    most: int
    handle: Optional[int] = None   # of the stream that begin made them on


class Cache8:
    """Keys and values of `layers` layers in `n_pages` pages of page_size tokens, 8-bit
    codes with a scale for each scale_block tokens and head, for up to `rows`
    sequences of max_tokens.  inv_freq: rotary frequencies (float64, by default
    base 10000 over the whole head), amplitude and interleaved as for realq_rotary.

    Any stream: a call on a stream other than the current one (`stream`) starts
    after what the current stream holds and takes its memory from its own stream,
    and the current stream has to wait for it before it reads its results, as
    with any operator.  The calls run one after the other, whatever their streams.

    In a graph: `attend` can be captured with the buffers that it is given; `begin`
    brings host numbers in and cannot.  To replay tokens, `begin` each one outside,
    with as many new tokens as the captured step, and copy its starts and positions
    there.  Replays are ordered by their streams, which is the caller's part."""

    def __init__(self, layers: int, n_pages: int, rows: int, max_tokens: int, n_kv: int, head_dim: int, page_size: int = 64,
                 scale_block: int = 16, inv_freq: Optional[torch.Tensor] = None, amplitude: float = 1.0, interleaved: bool = False,
                 device="cuda"):
        shape = (layers, n_pages, n_kv, page_size)
        new = lambda *s, dtype: torch.zeros(s, dtype=dtype, device=device)  # noqa: E731
        codes = [torch.full((*shape, head_dim), 128, dtype=torch.uint8, device=device) for _ in range(2)]
        scales = [new(*shape[:3], page_size // scale_block, dtype=torch.float32) for _ in range(2)]
        self.cache = kv_cache(codes[0], codes[1], scales[0], scales[1])
        self._sizes = layers, n_kv, head_dim, self.cache.device
        max_pages = -(-max_tokens // page_size)
        self.used, self.lengths = new(n_pages, dtype=torch.int32), new(rows, dtype=torch.int32)
        self.tables = torch.full((rows, max_pages), -1, dtype=torch.int32, device=device)
        self.pages = kv_pages(self.used, self.tables, self.lengths)
        self.moved_to = new(n_pages, dtype=torch.int32)
        self.inv_freq = (realq_rotary_frequencies(head_dim) if inv_freq is None else inv_freq).to(device)
        self.amplitude, self.interleaved = amplitude, interleaved
        self._pages_ws = workspace(realq_pages_workspace_size(n_pages, rows, max_pages), device)
        # (its size depends on the GPU alone)
        self._attend_ws = workspace(realq_kv_attention_workspace_size(self.cache, rows, 1, n_kv), device)
        self._latest = torch.cuda.current_stream(self.used.device)   # the latest call's
        self._handle = self._latest.cuda_stream

    def _own(self):
        return (*self.cache.tensors, *self.pages.tensors, self.moved_to, self.inv_freq, self._pages_ws, self._attend_ws)

    def _begin(self, stream, *given: Optional[torch.Tensor]):
        """A call on `stream` (None: the current one) begins: after the caller's work
        and the cache's latest call.  The context that it runs in."""
        handle = _stream(stream)
        if stream is None or handle == _stream(None):   # the current stream
            # (nothing to order, or nothing that a capture could; making stream objects would take as long as a small kernel)
            if handle == self._handle or torch.cuda.is_current_stream_capturing():
                return _HERE
        caller = torch.cuda.current_stream(self.used.device)
        s = caller if stream is None else stream
        kept = given
        if handle != self._handle:
            s.wait_stream(self._latest)
            self._latest, self._handle = s, handle
            kept += self._own()
        if s != caller:
            s.wait_stream(caller)
        for t in kept:   # not to be handed on before the call is done with it
            if isinstance(t, torch.Tensor):
                t.record_stream(s)
        return torch.cuda.stream(s)

    def _ints(self, rows: Rows) -> torch.Tensor:
        if isinstance(rows, torch.Tensor):
            return rows
        # (from pinned memory, which torch keeps until the copy is done: the host does not wait for the stream)
        return torch.tensor(list(rows), dtype=torch.int32, pin_memory=True).to(self.used.device, non_blocking=True)

    def begin(self, counts: Sequence[int], stream=None) -> Step:
        """Room for counts[s] new tokens in each row."""
        if len(counts) != self.tables.shape[0] or min(counts) < 0:
            raise ValueError(f"counts: {self.tables.shape[0]} numbers from 0 on expected")
        at = [0]
        for n in counts:
            at.append(at[-1] + n)
        with self._begin(stream):
            step = Step(self._ints(at), torch.empty(at[-1], dtype=torch.int64, device=self.used.device), max(counts), _stream(None))
            realq_pages_reserve(self.pages, step.starts, step.positions, self.cache, ws=self._pages_ws)
        return step

    def attend(self, step: Step, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, window: int = 0,
               scale: Optional[float] = None, stream=None) -> torch.Tensor:
        """The step's tokens through one layer: q and k get their positions (in place),
        k and v go into the cache, and q attends to all of its row's tokens so far.  (By the
        rows' latest lengths: a row takes part in the next step when all layers are through this one.)"""
        T, H, _ = q.shape
        if T != step.positions.shape[0]:
            raise ValueError(f"q: {step.positions.shape[0]} tokens expected, got {T}")
        self._refuse(layer, q, k, v, out, lse, window, scale)
        with self._begin(stream, q, k, v, out, lse, step.starts, step.positions):
            if step.handle not in (None, self._handle) and not torch.cuda.is_current_stream_capturing():
                for t in (step.starts, step.positions):   # (another step has come between)
                    t.record_stream(self._latest)
            if out is None:
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            if T == 0:
                return out
            realq_rotary(q, step.positions, self.inv_freq, q, k=k, k_out=k, interleaved=self.interleaved, amplitude=self.amplitude)
            realq_kv_append(self.cache, layer, k, v, step.starts, step.positions, self.tables)
            return realq_kv_attention(q, self.cache, layer, step.starts, self.lengths, self.tables, out, lse=lse, scale=scale,
                                      window=window, max_new=step.most, ws=self._attend_ws)

    def _refuse(self, layer, q, k, v, out, lse, window, scale) -> None:
        """What appending and attention would refuse, before q and k are turned."""
        layers, kv, head_dim, device = self._sizes
        dt, (T, H, D) = q.dtype, q.shape
        if not 0 <= layer < layers:
            raise ValueError(f"layer: one of {layers} expected, got {layer}")
        if D != head_dim or H % kv or not 0 < H <= 1024 * kv:
            raise ValueError(f"q: heads of {head_dim} values expected, 1 to 1024 for each of {kv}")
        if k.dtype is not dt or v.dtype is not dt:
            raise ValueError("q, k and v have one dtype")
        for t, name in ((k, "k"), (v, "v")):
            if t.shape != (T, kv, D) or t.get_device() != device or not t.is_contiguous():
                _, ld, hs = _heads(t, name, device, (T, kv, D))
                if min(ld, hs) < D:
                    raise ValueError(f"{name}: heads or tokens overlap")
        if out is not None:
            _buffer(out, q.shape, "out", device, dt)
        if lse is not None:
            _buffer(lse, (T, H), "lse", device, torch.float32)
        if window < 0 or (scale is not None and not abs(scale) <= 2.0 ** 127):
            raise ValueError("window from 0 on, |scale| up to 2^127 expected")

    def fork(self, src: Rows, dst: Rows, stream=None) -> None:
        """Rows dst[i] go on from rows src[i]'s sequences, all at once (a beam search's reordering)."""
        with self._begin(stream, src, dst):
            realq_pages_fork(self.pages, self._ints(src), self._ints(dst), ws=self._pages_ws)

    def release(self, rows: Rows, stream=None) -> None:
        """The rows' sequences leave."""
        with self._begin(stream, rows):
            realq_pages_release(self.pages, self._ints(rows))

    def compact(self, stream=None) -> torch.Tensor:
        """Pages in use to the front of the pool; each page's new number (-1: free)."""
        with self._begin(stream):
            realq_pages_compact(self.pages, self.cache, self.used, self.tables, self.moved_to, ws=self._pages_ws)
        return self.moved_to

    def check(self, stream=None) -> None:
        """Raises RealqError if a step since the last check found too few pages, or a bounded wait gave up (synchronizes).
        Where both happened, the latter is raised from the former.  What a wait that gave up left in the cache's
        workspace is cleared; the outputs since the last check are then unspecified."""
        error = None
        with self._begin(stream):
            for ws in (self._pages_ws, self._attend_ws):
                try:
                    realq_workspace_status(ws)
                except RealqError as e:
                    if e.status == REALQ_ERR_TIMEOUT:
                        ws.zero_()   # (arrival counters stay where the call left them)
                    e.__cause__, error = error, e
        if error is not None:
            raise error
