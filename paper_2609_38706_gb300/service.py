"""Convenience layer over the C-ABI: a device-resident key table plus
per-batch buffers, all allocated with PyTorch, every step run by libpk.

    kt = KeyTable(chunk_tokens=256, capacity_log2=20)
    d = kt.digests(descriptors)                  # a0: canonicalise + enc (host), SHA-256 (device)
    key_off, keys = kt.derive(tokens, tok_off, desc_idx, d)      # a1 + a2
    hit, slots = kt.lookup(keys, key_off)                        # a3
    result, slot_out = kt.store(keys, new_slots, key_off, hit)   # a4 (the misses)

A table or pool made with a stream runs on it, with the buffers that it makes;
device tensors that a caller passes, and reads of what it gets, the caller orders.
"""
from __future__ import annotations

import contextlib
import operator
from typing import Optional

import numpy as np
import torch

from . import pk


_NP_SIGNED = {torch.int32: np.int32, torch.int64: np.int64, torch.uint8: np.uint8}


def _stream(stream):
    """The torch stream of `stream`, a torch stream or a raw handle."""
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream))


def _on(stream):
    """Context in which PyTorch's work and allocations belong to `stream` (None: the current one)."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(_stream(stream))


def _dev(x, dtype, device, stream=None) -> torch.Tensor:
    """Host array or tensor -> contiguous device tensor of ``dtype``; unsigned
    host arrays of the same width are reinterpreted, not converted.  The copy is
    made on the current stream (one from the host is over when this returns);
    ``stream``, whose kernels will read it, is ordered behind it, and the copy's
    memory is not given out again before those have run."""
    if isinstance(x, torch.Tensor):
        t = x.to(device=device, dtype=dtype).contiguous()
    else:
        a = np.ascontiguousarray(x)
        want = np.dtype(_NP_SIGNED[dtype])
        a = a.view(want) if a.dtype.itemsize == want.itemsize and a.dtype.kind in "ui" else a.astype(want)
        t = torch.from_numpy(a).to(device=device)
    if stream is not None and t is not x:
        if isinstance(x, torch.Tensor) and x.is_cuda:
            _stream(stream).wait_stream(torch.cuda.current_stream(t.device))
        t.record_stream(_stream(stream))
    return t


def _empty(like: torch.Tensor, stream, *wanted) -> list:
    """Buffers (shape, dtype) on like's device that belong to `stream` (None: the current one), so that one freed while
    its kernel still runs is only given out again to later work of that stream."""
    device = like.device
    if stream is None:
        return [torch.empty(shape, dtype=dtype, device=device) for shape, dtype in wanted]
    with _on(stream):
        return [torch.empty(shape, dtype=dtype, device=device) for shape, dtype in wanted]


class KeyTable:
    def __init__(self, chunk_tokens: int, capacity_log2: int, max_probe: int = 0, device="cuda",
                 stream: Optional[torch.cuda.Stream] = None):
        self.device = torch.device(device)
        self.stream = stream
        self.chunk_tokens = int(chunk_tokens)
        self.capacity_log2 = int(capacity_log2)
        nbytes = pk.pk_table_bytes(capacity_log2)
        if nbytes == 0:
            raise pk.PKError(pk.PK_ERR_CAPACITY, "KeyTable")
        with _on(stream):
            self.table = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.ctx = pk.pk_init(self.table, chunk_tokens, capacity_log2, max_probe, stream)

    # -- lifecycle ---------------------------------------------------------
    def close(self):
        if self.ctx:
            torch.cuda.synchronize(self.device)
            pk.pk_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def entries(self) -> int:
        return pk.pk_entries(self.ctx, self.stream)

    def _new(self, shape, dtype, zero: bool = False) -> torch.Tensor:
        """A buffer that belongs to the table's stream."""
        with _on(self.stream):
            return (torch.zeros if zero else torch.empty)(shape, dtype=dtype, device=self.device)

    def save(self, dst: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Checkpoint the table (device tensor unless ``dst`` is given)."""
        if dst is None:
            dst = self._new(self.table.numel() + 64, torch.uint8)
        pk.pk_table_save(self.ctx, dst, self.stream)
        return dst

    def load(self, src: torch.Tensor) -> None:
        pk.pk_table_load(self.ctx, src, self.stream)

    def take_status(self) -> int:
        """Read and clear the device status word, behind all that was enqueued on its stream so far (synchronises)."""
        with _on(self.stream):
            v = int(self.status.item())
            self.status.zero_()
        return v

    def check(self, where: str = "device") -> None:
        v = self.take_status()
        if v != pk.PK_OK:
            raise pk.PKError(v, where)

    # -- steps -------------------------------------------------------------
    def digests(self, descriptors) -> torch.Tensor:
        enc, off = pk.pk_descriptors_encode(descriptors)
        D = off.size - 1
        enc_d = _dev(enc if enc.size else np.zeros(1, np.uint8), torch.uint8, self.device, self.stream)
        off_d = _dev(off, torch.int64, self.device, self.stream)
        out = self._new((max(D, 1), 32), torch.uint8, zero=True)
        pk.pk_digest_descriptors(self.ctx, enc_d[: enc.size], off_d, out, self.status, self.stream)
        return out[:D]

    def derive(self, tokens, tok_off, desc_idx, digests):
        tokens = _dev(tokens, torch.int32, self.device, self.stream)
        tok_off = _dev(tok_off, torch.int64, self.device, self.stream)
        desc_idx = _dev(desc_idx, torch.int32, self.device, self.stream)
        R = tok_off.numel() - 1
        cap = tokens.numel() // self.chunk_tokens
        key_off = self._new(R + 1, torch.int64)
        keys = self._new((max(cap, 0), 32), torch.uint8)
        pk.pk_derive_keys(self.ctx, tokens, tok_off, desc_idx, digests, key_off, keys, self.status, self.stream)
        return key_off, keys

    def derive_enc(self, tokens, tok_off, desc_idx, descriptors):
        """Descriptor digests and keys in one call (pk_derive_keys_enc)."""
        enc, off = pk.pk_descriptors_encode(descriptors)
        D = off.size - 1
        enc_d = _dev(enc if enc.size else np.zeros(1, np.uint8), torch.uint8, self.device, self.stream)[: enc.size]
        off_d = _dev(off, torch.int64, self.device, self.stream)
        digests = self._new((max(D, 1), 32), torch.uint8, zero=True)[:D]
        tokens = _dev(tokens, torch.int32, self.device, self.stream)
        tok_off = _dev(tok_off, torch.int64, self.device, self.stream)
        desc_idx = _dev(desc_idx, torch.int32, self.device, self.stream)
        R = tok_off.numel() - 1
        cap = tokens.numel() // self.chunk_tokens
        key_off = self._new(R + 1, torch.int64)
        keys = self._new((max(cap, 0), 32), torch.uint8)
        pk.pk_derive_keys_enc(self.ctx, tokens, tok_off, desc_idx, enc_d, off_d, digests, key_off, keys,
                              self.status, self.stream)
        return digests, key_off, keys

    def lookup(self, keys, key_off):
        R = key_off.numel() - 1
        hit = self._new(R, torch.int32)
        slots = self._new(keys.shape[0], torch.int32)
        pk.pk_lookup(self.ctx, keys, key_off, hit, slots, self.status, self.stream)
        return hit, slots

    def store(self, keys, slots, key_off=None, hit=None):
        """List mode (key_off is None) or miss-range mode (key_off and hit)."""
        if keys.shape[1] == 16:  # widen 16-byte prefixes to the 32-byte key stride
            k = self._new((keys.shape[0], 32), torch.uint8, zero=True)
            narrow = _dev(keys, torch.uint8, self.device, self.stream)
            with _on(self.stream):
                k[:, :16] = narrow
            keys = k
        else:
            keys = _dev(keys, torch.uint8, self.device, self.stream)
        slots = _dev(slots if isinstance(slots, torch.Tensor) else np.asarray(slots, np.uint32), torch.int32,
                     self.device, self.stream)
        n = keys.shape[0]
        result = self._new(n, torch.int32)
        slot_out = self._new(n, torch.int32)
        pk.pk_store(self.ctx, keys, slots, result, slot_out, self.status, key_off, hit, self.stream)
        return result, slot_out

    def lookup_store(self, keys, key_off, new_slots):
        """lookup followed by store of the miss ranges, in one pass: returns
        (hit, slots, result, slot_out) as the two calls would."""
        R = key_off.numel() - 1
        n = keys.shape[0]
        new_slots = _dev(new_slots if isinstance(new_slots, torch.Tensor) else np.asarray(new_slots, np.uint32),
                         torch.int32, self.device, self.stream)
        hit = self._new(R, torch.int32)
        slots = self._new(n, torch.int32)
        result = self._new(n, torch.int32)
        slot_out = self._new(n, torch.int32)
        pk.pk_lookup_store(self.ctx, keys, new_slots, key_off, hit, slots, result, slot_out, self.status,
                           self.stream)
        return hit, slots, result, slot_out

    def derive_lookup_store(self, tokens, tok_off, desc_idx, descriptors, new_slots):
        """The whole hot path in one call (pk_derive_lookup_store): returns
        (digests, key_off, keys, hit, slots, result, slot_out)."""
        enc, off = pk.pk_descriptors_encode(descriptors)
        D = off.size - 1
        enc_d = _dev(enc if enc.size else np.zeros(1, np.uint8), torch.uint8, self.device, self.stream)[: enc.size]
        off_d = _dev(off, torch.int64, self.device, self.stream)
        digests = self._new((max(D, 1), 32), torch.uint8, zero=True)[:D]
        tokens = _dev(tokens, torch.int32, self.device, self.stream)
        tok_off = _dev(tok_off, torch.int64, self.device, self.stream)
        desc_idx = _dev(desc_idx, torch.int32, self.device, self.stream)
        R = tok_off.numel() - 1
        cap = tokens.numel() // self.chunk_tokens
        key_off = self._new(R + 1, torch.int64)
        keys = self._new((max(cap, 0), 32), torch.uint8)
        new_slots = _dev(new_slots if isinstance(new_slots, torch.Tensor) else np.asarray(new_slots, np.uint32),
                         torch.int32, self.device, self.stream)
        hit = self._new(R, torch.int32)
        slots = self._new(max(cap, 0), torch.int32)
        result = self._new(max(cap, 0), torch.int32)
        slot_out = self._new(max(cap, 0), torch.int32)
        pk.pk_derive_lookup_store(self.ctx, tokens, tok_off, desc_idx, enc_d, off_d, digests, key_off, keys, new_slots,
                                  hit, slots, result, slot_out, self.status, self.stream)
        return digests, key_off, keys, hit, slots, result, slot_out

    # -- budget mode (eviction under a fixed budget) -------------------------
    def attach_stamps(self) -> torch.Tensor:
        """Turn budget mode on: a zeroed last-use stamp per entry, and the
        scratch and output buffers of evict()."""
        cap = 1 << self.capacity_log2
        self.stamps = self._new(pk.pk_stamps_bytes(self.capacity_log2) // 8, torch.int64)
        pk.pk_attach_stamps(self.ctx, self.stamps, self.stream)
        self.evict_scratch = self._new(pk.pk_evict_scratch_bytes(self.capacity_log2), torch.uint8)
        self.evicted = self._new(cap, torch.int32)
        self.n_evicted = self._new(1, torch.int64, zero=True)
        return self.stamps

    def evict(self, budget: int, keep: int):
        """Enqueue pk_evict; returns (evicted slots buffer, count tensor),
        valid up to the count once the stream has run."""
        pk.pk_evict(self.ctx, budget, keep, self.evict_scratch, self.evicted, self.n_evicted, self.status,
                    self.stream)
        return self.evicted, self.n_evicted

    def seed(self, seed_keys, filler, target_entries: int) -> int:
        """Pre-fill: seed keys in order (slot = list index), then filler keys
        (continuing the index) until the table holds target_entries entries."""
        n_seed = int(seed_keys.shape[0])
        if n_seed:
            self.store(seed_keys, np.arange(n_seed, dtype=np.uint32))
        need = target_entries - self.entries()
        if need > 0:
            self.store(filler[:need], np.arange(n_seed, n_seed + need, dtype=np.uint32))
        self.check("seed")
        return self.entries()


def _limits(where: str, window: Optional[int], sinks: int):
    """(window, sinks) as the library takes them: 0 is no window."""
    if window is not None and window < 1:
        raise pk.PKError(pk.PK_ERR_ARG, where + ": a window holds a query's own position at least")
    return 0 if window is None else operator.index(window), operator.index(sinks)


class KVPages:
    """What the slots of a KeyTable point at: a pool of KV pages held in 4 bits
    (layout and format: pk.h), with its calls.  Page tables are int32
    [R, page_stride] tensors of (uint32) slots, one row a request.

        kv = KVPages(n_slots, page_tokens=kt.chunk_tokens, kv_heads=8, head_dim=128)
        kv.write(k, v, tok_off, start, pages)          # the misses' chunks, or a decode step's tokens
        k, v = kv.read(tok_off, start, pages, n)       # a hit's prefix
        out, lse = kv.attend_prompt(q, k, v, q_off, k_off)
        out, lse = kv.attend(q, kv_len, pages, scale, weight=weight)
        pages, weight, kv_len, _ = kv.evict(pages, weight, kv_len, budget, sinks, recent)
        kv.check()                                     # any call's device error

    Bind ``kv.kv_format`` in the descriptors of what is stored here.  With ``stream`` the pool's zero fill, every call and
    the status word belong to that stream; tensors that the caller passes, ``pool`` among them, the caller orders."""

    def __init__(self, n_slots: int, page_tokens: int, kv_heads: int, head_dim: int, k_scale: float = 1.0,
                 v_scale: float = 1.0, device="cuda", stream: Optional[torch.cuda.Stream] = None,
                 pool: Optional[torch.Tensor] = None):
        self.stream = stream
        self.page_tokens, self.kv_heads, self.head_dim = int(page_tokens), int(kv_heads), int(head_dim)
        nbytes = pk.pk_kv_page_bytes(page_tokens, kv_heads, head_dim) if min(page_tokens, kv_heads, head_dim) > 0 else 0
        if nbytes == 0 or n_slots < 1:
            raise pk.PKError(pk.PK_ERR_ARG, "KVPages")
        if pool is None:
            with _on(stream):
                pool = torch.zeros((n_slots, nbytes), dtype=torch.uint8, device=device)
        if pool.dtype != torch.uint8 or not pool.is_contiguous() or pool.numel() != n_slots * nbytes or not pool.is_cuda:
            raise pk.PKError(pk.PK_ERR_ARG, "KVPages: pool is contiguous uint8 [n_slots, pk_kv_page_bytes] on the device")
        self.pool, self.device = pool, pool.device
        with _on(stream):
            self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._scratch_bytes: dict = {}
        self.kv = pk.pk_kv_cache(pool.data_ptr(), n_slots, page_tokens, kv_heads, head_dim, k_scale, v_scale)
        self.kv.device = self.device.index

    @property
    def kv_format(self) -> str:
        """The descriptor's kv_format for pages of this pool: format, block and tensor scales."""
        return f"fp4_e2m1_b16_e4m3:k={self.kv.k_scale!r}:v={self.kv.v_scale!r}"

    take_status, check = KeyTable.take_status, KeyTable.check

    def write(self, k, v, tok_off, start, pages) -> None:
        pk.pk_kv_write(self.kv, k, v, tok_off, start, pages, self.status, self.stream)

    def read(self, tok_off, start, pages, n_tokens: int, dtype=torch.bfloat16):
        """(k, v) [n_tokens, kv_heads, head_dim]; rows that belong to no request are unspecified."""
        shape = (n_tokens, self.kv_heads, self.head_dim)
        k, v = _empty(self.pool, self.stream, (shape, dtype), (shape, dtype))
        pk.pk_kv_read(self.kv, k, v, tok_off, start, pages, self.status, self.stream)
        return k, v

    def attend(self, q, kv_len, pages, scale: Optional[float] = None, weight: Optional[torch.Tensor] = None,
               window: Optional[int] = None, sinks: int = 0):
        """q [R, n_q, q_heads, head_dim] over the pages: (out like q, lse float32 [R, n_q, q_heads]).  weight
        (float32, like pages) gets each page's attention weight added.  With ``window`` a query at position p sees the
        positions above p - window, and the first ``sinks`` ones; pages out of sight are not read."""
        if q.dim() != 4:
            raise pk.PKError(pk.PK_ERR_ARG, "KVPages.attend: q is [R, n_q, q_heads, head_dim]")
        R, n_q, heads, D = q.shape
        limits = _limits("KVPages.attend", window, sinks)
        key = (R, n_q, heads, pages.shape[-1], weight is not None, *limits)
        nbytes = self._scratch_bytes.get(key)
        if nbytes is None:
            if len(self._scratch_bytes) >= 4096:
                self._scratch_bytes.clear()
            nbytes = self._scratch_bytes[key] = pk.pk_attend_cache_window_scratch_bytes(self.kv, *key)
        out, lse, scratch = _empty(q, self.stream, (q.shape, q.dtype), (q.shape[:3], torch.float32),
                                   ((nbytes,), torch.uint8))
        scale = D ** -0.5 if scale is None else scale
        if limits[0]:
            pk.pk_attend_cache_window(self.kv, q, out, lse, n_q, kv_len, pages, scale, *limits, weight, scratch, self.status,
                                      self.stream)
        else:
            pk.pk_attend_cache(self.kv, q, out, lse, n_q, kv_len, pages, scale, weight, scratch, self.status, self.stream)
        return out, lse

    def attend_chunk(self, q, q_off, kv_len, pages, scale: Optional[float] = None, window: Optional[int] = None,
                     sinks: int = 0):
        """Chunks of new tokens, written before, over the pages: q [n_q, q_heads, head_dim], request r's rows q_off[r] ..
        q_off[r + 1] at its last positions: (out like q, lse float32 [n_q, q_heads]).  ``window`` and ``sinks`` as in
        attend.  One very long request among many short ones is faster in a call of its own."""
        if q.dim() != 3:
            raise pk.PKError(pk.PK_ERR_ARG, "KVPages.attend_chunk: q is [n_q, q_heads, head_dim]")
        n_q, heads, D = q.shape
        limits = _limits("KVPages.attend_chunk", window, sinks)
        key = (q.dtype, n_q, pages.shape[0], heads, pages.shape[-1], *limits)
        nbytes = self._scratch_bytes.get(key)
        if nbytes is None:
            if len(self._scratch_bytes) >= 4096:
                self._scratch_bytes.clear()
            nbytes = self._scratch_bytes[key] = pk.pk_attend_chunk_scratch_bytes(self.kv, *key)
        out, lse, scratch = _empty(q, self.stream, (q.shape, q.dtype), (q.shape[:2], torch.float32),
                                   ((nbytes,), torch.uint8))
        pk.pk_attend_chunk(self.kv, q, out, lse, q_off, kv_len, pages, D ** -0.5 if scale is None else scale, *limits, scratch,
                           self.status, self.stream)
        return out, lse

    def rotate(self, q, k, tok_off, start, rotary, q_weight=None, k_weight=None, eps: float = 1e-6, out=None):
        """rotate on the pool's stream, its device errors in the pool's status word: what write() and attend() take."""
        return rotate(q, k, tok_off, start, rotary, q_weight, k_weight, eps, out, self.status, self.stream)

    def attend_prompt(self, q, k, v, q_off, k_off, scale: Optional[float] = None):
        """attend_prompt on the pool's stream, its device errors in the pool's status word."""
        return attend_prompt(q, k, v, q_off, k_off, scale, self.status, self.stream)

    def evict(self, pages, weight, kv_len, budget: int, sinks: int, recent: int):
        """evict_pages for pages of this pool, on its stream, its device errors in the pool's status word."""
        return evict_pages(pages, weight, kv_len, self.page_tokens, budget, sinks, recent, self.status, self.stream)


class Rotary:
    """How positions rotate a head's first ``rotary_dim`` dimensions (pk_rotary): pair i, of dimensions (i, i +
    rotary_dim/2) or, ``interleaved``, (2i, 2i + 1), by ``base ** (-2 i / rotary_dim)`` radians a position.  For longer
    contexts than a model was made for these are divided by ``factor``: all of them, or with ``context``, its own context,
    by parts; ``amplitude`` multiplies what was rotated.  The parts' ramp runs over a pair's turns in that context
    (pk_rotary_turns), or with ``ramp="index"`` over its index, between rounded ends (pk_rotary_turns_by_index): the angles
    differ much, and a model takes those that it was tuned with.  ``turns`` (uint64 [rotary_dim / 2], fractions of a turn by
    2^64) takes the place of base and factor.

    The table is copied to ``device`` once, and that copy is over when the object exists.  Its memory is not given out again
    before the calls that read it have run, on whatever stream."""

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, base: float = 10000.0, interleaved: bool = False,
                 factor: float = 1.0, context: Optional[float] = None, low: float = 1.0, high: float = 32.0,
                 amplitude: float = 1.0, turns=None, device="cuda", ramp: str = "turns"):
        self.head_dim, self.rotary_dim = int(head_dim), int(head_dim if rotary_dim is None else rotary_dim)
        if self.rotary_dim < 16 or self.rotary_dim % 16 or self.rotary_dim > self.head_dim or not np.isfinite(amplitude):
            raise pk.PKError(pk.PK_ERR_ARG, "Rotary: rotary_dim is a multiple of 16, up to head_dim; amplitude is finite")
        if ramp not in ("turns", "index"):
            raise pk.PKError(pk.PK_ERR_ARG, "Rotary: the ramp is over turns or index")
        if turns is None:
            make = pk.pk_rotary_turns if ramp == "turns" else pk.pk_rotary_turns_by_index
            turns = make(self.rotary_dim, base, factor, context or 0.0, low, high)
        turns = np.ascontiguousarray(turns)
        if turns.dtype != np.uint64 or turns.shape != (self.rotary_dim // 2,):
            raise pk.PKError(pk.PK_ERR_ARG, "Rotary: turns is uint64 [rotary_dim / 2]")
        self.turns = torch.from_numpy(turns.view(np.int64)).to(device)
        self.made_on = pk._stream_of(None, self.turns) if self.turns.is_cuda else None
        self.table = pk.pk_rotary(self.turns.data_ptr(), self.rotary_dim, int(bool(interleaved)), amplitude)


def rotate(q, k, tok_off, start, rotary: Rotary, q_weight: Optional[torch.Tensor] = None,
           k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, out=None, status: Optional[torch.Tensor] = None,
           stream=None):
    """Norms of queries and keys by head (where weights are given) and their rotation, in one pass (pk_rotate): (q, k),
    new tensors or ``out``, a pair that may be (q, k) themselves.  q [tokens, q_heads, D], k [tokens, kv_heads, D]; token i
    of request r, row tok_off[r] + i, has position start[r] + i, where KVPages.write puts it.  Rows that belong to no
    request are unspecified in new tensors, and stay as they are in ``out``.  ``status`` as in attend_prompt
    (KVPages.rotate passes the pool's)."""
    if q.shape[-1] != rotary.head_dim or rotary.turns.device != q.device:
        raise pk.PKError(pk.PK_ERR_ARG, "rotate: rotary is for other heads, or on another device")
    q_out, k_out = out if out is not None else _empty(q, stream, (q.shape, q.dtype), (k.shape, k.dtype))
    if pk._stream_of(stream, rotary.turns) != rotary.made_on:  # the table belongs to the stream that it was made on
        rotary.turns.record_stream(torch.cuda.current_stream(rotary.turns.device) if stream is None else _stream(stream))
    pk.pk_rotate(q, k, q_out, k_out, rotary.table, q_weight, k_weight, eps, tok_off, start, status, stream)
    return q_out, k_out


def attend_prompt(q, k, v, q_off, k_off, scale: Optional[float] = None, status: Optional[torch.Tensor] = None,
                  stream=None):
    """Causal attention over packed prompts (pk_attend_prompt): (out like q, lse float32 [n_q, q_heads]).  Device errors
    go to ``status`` (int32, zeroed by the caller; KVPages.attend_prompt passes the pool's); without one the caller
    answers for the offsets: what is wrong with them leaves the outputs unspecified and is not reported."""
    nbytes = pk.pk_attend_prompt_scratch_bytes(max(q_off.numel() - 1, 0))
    out, lse, scratch = _empty(q, stream, (q.shape, q.dtype), (q.shape[:2], torch.float32), ((nbytes,), torch.uint8))
    pk.pk_attend_prompt(q, k, v, out, lse, q_off, k_off, q.shape[-1] ** -0.5 if scale is None else scale, scratch,
                        status, stream)
    return out, lse


def evict_pages(pages, weight, kv_len, page_tokens: int, budget: int, sinks: int, recent: int,
                status: Optional[torch.Tensor] = None, stream=None):
    """Cut each request to `budget` pages by accumulated attention weight (pk_evict_pages): (pages [R, budget],
    weight [R, budget], kv_len [R], evicted slots like pages), unused places PK_NO_SLOT (-1) and 0.  ``status`` as in
    attend_prompt (KVPages.evict passes the pool's)."""
    kept = (pages.shape[0], max(budget, 0))
    pages_out, weight_out, kv_len_out, evicted = _empty(
        pages, stream, (kept, torch.int32), (kept, torch.float32), (kept[:1], torch.int32), (pages.shape, torch.int32))
    pk.pk_evict_pages(pages, weight, kv_len, page_tokens, budget, sinks, recent, pages_out, weight_out, kv_len_out,
                      evicted, status, stream)
    return pages_out, weight_out, kv_len_out, evicted


def u32(t: torch.Tensor) -> np.ndarray:
    """int32 device tensor holding uint32 values -> numpy uint32."""
    return t.cpu().numpy().view(np.uint32)
