"""Thin Python binding of libpk (include/pk.h).

Argument marshalling only: every function has the name of the C entry point
it calls, turns tensors into raw pointers and sizes, passes the CUDA stream
handle, and raises ``PKError`` on a negative status.  All computation happens
in the library's CUDA kernels (and its host canonicaliser); there is no
fallback: if ``libpk.so`` has not been built this module raises on first use.
"""
from __future__ import annotations

import ctypes
import os
from typing import Iterable, Mapping, Optional, Sequence

import numpy as np
import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_build", "libpk.so")

PK_OK = 0
PK_ERR_ARG = -1
PK_ERR_CAPACITY = -2
PK_ERR_UNRESOLVED = -3
PK_ERR_FIELD_TOO_LONG = -4
PK_ERR_TABLE_FULL = -5
PK_ERR_PROBE_LIMIT = -6
PK_ERR_RESERVED_KEY = -7
PK_ERR_CUDA = -8
PK_ERR_TOO_LARGE = -9
PK_ERR_TIMEOUT = -10
PK_PAGE_ABSENT, PK_PAGE_EQUAL, PK_PAGE_DIFFERS = 0, 1, 2
PK_NOALLOC_MAX_ENTRIES = 1 << 18
PK_STORE_SKIPPED = 0
PK_STORE_INSERTED = 1
PK_STORE_PRESENT = 2
PK_NO_SLOT = 0xFFFFFFFF
PK_KEY_BYTES = 32
PK_ENTRY_BYTES = 32
PK_KEY_STRING_CHARS = 22
PK_KEY_STRING_MAX_WIDTH = 256
PK_BF16, PK_FP16 = 0, 1
REGISTRY_V1 = ("model_id", "weight_precision", "weight_version", "adapter_id", "kv_format", "salt")


class PKError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {pk_strerror(code)} ({code})")
        self.code = code


class pk_bytes(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("len", ctypes.c_uint32)]


class pk_descriptor(ctypes.Structure):
    _fields_ = [(name, pk_bytes) for name in REGISTRY_V1] + [
        ("extra", ctypes.POINTER(pk_bytes)), ("n_extra", ctypes.c_uint32)]


class pk_config(ctypes.Structure):
    _fields_ = [("chunk_tokens", ctypes.c_uint32), ("capacity_log2", ctypes.c_uint32),
                ("max_probe", ctypes.c_uint32), ("table_dev", ctypes.c_void_p),
                ("table_bytes", ctypes.c_size_t)]


class pk_kv_cache(ctypes.Structure):
    _fields_ = [("pool_dev", ctypes.c_void_p), ("n_slots", ctypes.c_uint64), ("page_tokens", ctypes.c_uint32),
                ("kv_heads", ctypes.c_uint32), ("head_dim", ctypes.c_uint32), ("k_scale", ctypes.c_float),
                ("v_scale", ctypes.c_float)]
    device: Optional[int] = None  # index of the pool's device, where known


class pk_heads(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("tok_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


_lib = None
_VP, _U32, _U64, _I32 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int32


def lib() -> ctypes.CDLL:
    """Load libpk.so (built by ``__graft_entry__.build()``); raise if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"libpk.so not found at {_LIB_PATH}: build it first "
                               "(python -c 'import __graft_entry__ as g; g.build()')")
        L = ctypes.CDLL(_LIB_PATH)
        sig = {
            "pk_table_bytes": (ctypes.c_size_t, [_U32]),
            "pk_init": (ctypes.c_int, [ctypes.POINTER(_VP), ctypes.POINTER(pk_config), _VP]),
            "pk_destroy": (ctypes.c_int, [_VP]),
            "pk_descriptor_encode": (ctypes.c_int, [ctypes.POINTER(pk_descriptor), _VP, ctypes.c_size_t,
                                                    ctypes.POINTER(ctypes.c_size_t)]),
            "pk_descriptors_encode": (ctypes.c_int, [ctypes.POINTER(pk_descriptor), _U32, _VP,
                                                     ctypes.c_size_t, _VP]),
            "pk_descriptor_digest": (ctypes.c_int, [ctypes.POINTER(pk_descriptor), _VP]),
            "pk_worker_digest": (ctypes.c_int, [ctypes.POINTER(pk_descriptor), _VP]),
            "pk_request_digest": (ctypes.c_int, [_VP, ctypes.POINTER(pk_descriptor), _VP]),
            "pk_request_digests": (ctypes.c_int, [_VP, ctypes.POINTER(pk_descriptor), _U32, _VP]),
            "pk_digest_descriptors": (ctypes.c_int, [_VP, _VP, _U64, _VP, _U32, _VP, _VP, _VP]),
            "pk_derive_keys": (ctypes.c_int, [_VP, _VP, _U64, _VP, _U32, _VP, _VP, _U32, _VP, _VP, _U64,
                                              _VP, _VP]),
            "pk_derive_keys_enc": (ctypes.c_int, [_VP, _VP, _U64, _VP, _U32, _VP, _VP, _U64, _VP, _U32, _VP, _VP, _VP,
                                                  _U64, _VP, _VP]),
            "pk_lookup": (ctypes.c_int, [_VP, _VP, _VP, _U32, _U64, _VP, _VP, _VP, _VP]),
            "pk_store": (ctypes.c_int, [_VP, _VP, _VP, _U64, _VP, _VP, _U32, _VP, _VP, _VP, _VP]),
            "pk_lookup_store": (ctypes.c_int, [_VP, _VP, _VP, _VP, _U32, _U64, _VP, _VP, _VP, _VP, _VP, _VP]),
            "pk_derive_lookup_store": (ctypes.c_int, [_VP, _VP, _U64, _VP, _U32, _VP, _VP, _U64, _VP, _U32, _VP, _VP,
                                                      _VP, _U64, _VP, _VP, _VP, _VP, _VP, _VP, _VP]),
            "pk_entries": (ctypes.c_int, [_VP, ctypes.POINTER(ctypes.c_uint64), _VP]),
            "pk_store_noalloc": (ctypes.c_int, [ctypes.POINTER(pk_config), _VP, _VP, _U64, _VP, _VP, _U32, _VP, _VP,
                                                _VP, _VP]),
            "pk_compare_pages": (ctypes.c_int, [_VP, _VP, _VP, _U64, _U64, _U64, _VP, _VP, _VP, _VP]),
            "pk_content_scratch_bytes": (ctypes.c_size_t, [_U64]),
            "pk_content_digest": (ctypes.c_int, [_VP, _U64, _VP, ctypes.c_size_t, _VP, _VP]),
            "pk_content_scratch_bytes_batch": (ctypes.c_size_t, [_VP, _U32]),
            "pk_content_digests": (ctypes.c_int, [_VP, _VP, _U32, _VP, ctypes.c_size_t, _VP, _VP]),
            "pk_tensor_identity": (ctypes.c_int, [ctypes.POINTER(pk_bytes), ctypes.POINTER(pk_bytes), _VP, _U32,
                                                  _U64, _VP, _VP]),
            "pk_adapter_identity": (ctypes.c_int, [_VP, _U32, ctypes.POINTER(pk_bytes), _U32, _VP]),
            "pk_stamps_bytes": (ctypes.c_size_t, [_U32]),
            "pk_attach_stamps": (ctypes.c_int, [_VP, _VP, ctypes.c_size_t, _VP]),
            "pk_evict_scratch_bytes": (ctypes.c_size_t, [_U32]),
            "pk_evict": (ctypes.c_int, [_VP, _U64, _U64, _VP, ctypes.c_size_t, _VP, _U64, _VP, _VP, _VP]),
            "pk_evict_barrier_timeout_test": (ctypes.c_int, [_VP, _U64, _VP, ctypes.c_size_t, _U32, _VP, _VP]),
            "pk_key_string": (ctypes.c_int, [_VP, _VP]),
            "pk_model_tag": (ctypes.c_int, [ctypes.POINTER(pk_descriptor), _VP]),
            "pk_key_strings": (ctypes.c_int, [_VP, _U64, _VP, _U32, _U32, _VP, _VP]),
            "pk_table_save": (ctypes.c_int, [_VP, _VP, ctypes.c_size_t, _VP]),
            "pk_table_load": (ctypes.c_int, [_VP, _VP, ctypes.c_size_t, _VP]),
            "pk_kv_page_bytes": (ctypes.c_size_t, [_U32, _U32, _U32]),
            "pk_kv_write": (ctypes.c_int, [_VP, _U32, _VP, _VP, _U64, _VP, _VP, _U32, _VP, _U64, _VP, _VP]),
            "pk_kv_read": (ctypes.c_int, [_VP, _U32, _VP, _VP, _U64, _VP, _VP, _U32, _VP, _U64, _VP, _VP]),
            "pk_attend_prompt_scratch_bytes": (ctypes.c_size_t, [_U32]),
            "pk_attend_prompt": (ctypes.c_int, [_U32, _VP, _VP, _VP, _VP, _VP, _U64, _U64, _VP, _VP, _U32, _U32, _U32,
                                                _U32, ctypes.c_float, _VP, ctypes.c_size_t, _VP, _VP]),
            "pk_attend_cache_scratch_bytes": (ctypes.c_size_t, [_VP, _U32, _U32, _U32, _U64, ctypes.c_int]),
            "pk_attend_cache": (ctypes.c_int, [_VP, _U32, _VP, _VP, _VP, _U32, _U32, _U32, ctypes.c_float, _VP, _VP,
                                               _U64, _VP, _VP, ctypes.c_size_t, _VP, _VP]),
            "pk_evict_pages": (ctypes.c_int, [_VP, _VP, _VP, _U32, _U64, _U32, _U32, _U32, _U32, _VP, _VP, _VP, _VP,
                                              _VP, _VP]),
            "pk_strerror": (ctypes.c_char_p, [ctypes.c_int]),
        }
        for name, (res, args) in sig.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def _check(rc: int, where: str) -> None:
    if rc != PK_OK:
        raise PKError(rc, where)


if hasattr(torch._C, "_cuda_getDevice"):  # without what a public call adds to it, as every call asks

    def _current_device() -> int:
        """Index of the device that kernels are launched on.  Only asked where CUDA is in use."""
        return torch._C._cuda_getDevice()
else:
    _current_device = torch.cuda.current_device


def _p(t) -> Optional[int]:
    """Raw pointer of a tensor / ndarray (None for None).  A device tensor is on the current device."""
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        if t.is_cuda and t.get_device() != _current_device():
            raise PKError(PK_ERR_ARG, "a tensor is on another device than the current one")
        return t.data_ptr() if t.numel() else None
    if isinstance(t, np.ndarray):
        return t.ctypes.data if t.size else None
    return int(t)


def _s(stream) -> Optional[int]:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


class Descriptors:
    """ctypes array of pk_descriptor built from dicts (field name -> str/bytes,
    optional ``extra`` list), keeping the byte buffers alive."""

    def __init__(self, descs: Iterable[Mapping]):
        descs = list(descs)
        self._keep = []
        self.array = (pk_descriptor * max(len(descs), 1))()
        self.count = len(descs)
        for j, d in enumerate(descs):
            for name in REGISTRY_V1:
                setattr(self.array[j], name, self._b(d.get(name, b"")))
            extra = list(d.get("extra", ()) or ())
            if extra:
                arr = (pk_bytes * len(extra))(*[self._b(x) for x in extra])
                self._keep.append(arr)
                self.array[j].extra = ctypes.cast(arr, ctypes.POINTER(pk_bytes))
                self.array[j].n_extra = len(extra)

    def _b(self, v) -> pk_bytes:
        if v is None:
            v = b""
        if isinstance(v, str):
            v = v.encode("utf-8")
        v = bytes(v)
        buf = ctypes.create_string_buffer(v, len(v) + 1)
        self._keep.append(buf)
        return pk_bytes(ctypes.cast(buf, ctypes.c_void_p), len(v))


def _descs(d) -> Descriptors:
    return d if isinstance(d, Descriptors) else Descriptors(d)


# ---------------------------------------------------------------------------
# entry points
# ---------------------------------------------------------------------------
def pk_strerror(code: int) -> str:
    try:
        return lib().pk_strerror(code).decode()
    except RuntimeError:
        return f"status {code}"


def pk_table_bytes(capacity_log2: int) -> int:
    return int(lib().pk_table_bytes(capacity_log2))


def pk_init(table: torch.Tensor, chunk_tokens: int, capacity_log2: int, max_probe: int = 0,
            stream=None) -> int:
    """Bind a caller-owned table tensor (>= pk_table_bytes bytes) and clear it.
    Returns the opaque context pointer."""
    cfg = pk_config(chunk_tokens, capacity_log2, max_probe, _p(table),
                    table.numel() * table.element_size())
    out = ctypes.c_void_p()
    _check(lib().pk_init(ctypes.byref(out), ctypes.byref(cfg), _s(stream)), "pk_init")
    return out.value


def pk_destroy(ctx: int) -> None:
    _check(lib().pk_destroy(ctx), "pk_destroy")


def pk_descriptor_encode(desc) -> bytes:
    d = _descs([desc]) if isinstance(desc, Mapping) else _descs(desc)
    n = ctypes.c_size_t(0)
    rc = lib().pk_descriptor_encode(d.array, None, 0, ctypes.byref(n))
    if rc not in (PK_OK, PK_ERR_ARG):
        _check(rc, "pk_descriptor_encode")
    buf = ctypes.create_string_buffer(max(n.value, 1))
    _check(lib().pk_descriptor_encode(d.array, buf, n.value, ctypes.byref(n)), "pk_descriptor_encode")
    return buf.raw[: n.value]


def pk_descriptors_encode(descs, out: Optional[np.ndarray] = None,
                          enc_off: Optional[np.ndarray] = None) -> tuple[np.ndarray, np.ndarray]:
    """Encode D descriptors into ``out`` (uint8, host; pinned tensors welcome)
    and ``enc_off`` (int64[D+1]).  Returns views (bytes used, offsets)."""
    d = _descs(descs)
    if out is None:
        out = np.zeros(64 * 1024 + d.count * (7 * 4 + 8 * 4096), np.uint8)
    if enc_off is None:
        enc_off = np.zeros(d.count + 1, np.int64)
    cap = out.numel() if isinstance(out, torch.Tensor) else out.size
    _check(lib().pk_descriptors_encode(d.array, d.count, _p(out), cap, _p(enc_off)), "pk_descriptors_encode")
    used = int(enc_off[d.count])
    return out[:used], enc_off


def pk_descriptor_digest(desc) -> bytes:
    d = _descs([desc]) if isinstance(desc, Mapping) else _descs(desc)
    out = (ctypes.c_uint8 * 32)()
    _check(lib().pk_descriptor_digest(d.array, out), "pk_descriptor_digest")
    return bytes(out)


def pk_worker_digest(desc) -> bytes:
    d = _descs([desc]) if isinstance(desc, Mapping) else _descs(desc)
    out = (ctypes.c_uint8 * 32)()
    _check(lib().pk_worker_digest(d.array, out), "pk_worker_digest")
    return bytes(out)


def pk_request_digest(worker: bytes, desc) -> bytes:
    d = _descs([desc]) if isinstance(desc, Mapping) else _descs(desc)
    w = (ctypes.c_uint8 * 32).from_buffer_copy(bytes(worker))
    out = (ctypes.c_uint8 * 32)()
    _check(lib().pk_request_digest(w, d.array, out), "pk_request_digest")
    return bytes(out)


def pk_request_digests(worker: bytes, descs) -> np.ndarray:
    """uint8[n][32]: pk_request_digest of each descriptor under one worker digest."""
    d = _descs(descs)
    w = (ctypes.c_uint8 * 32).from_buffer_copy(bytes(worker))
    out = np.zeros((max(d.count, 1), 32), np.uint8)
    _check(lib().pk_request_digests(w, d.array, d.count, _p(out)), "pk_request_digests")
    return out[: d.count]


def two_level_digests(descs) -> np.ndarray:
    """uint8[D][32]: the two-level digest of each descriptor (its own worker
    half, then its request half)."""
    out = np.zeros((len(descs), 32), np.uint8)
    for j, d in enumerate(descs):
        out[j] = np.frombuffer(pk_request_digest(pk_worker_digest(d), d), np.uint8)
    return out


def pk_digest_descriptors(ctx: int, enc: torch.Tensor, enc_off: torch.Tensor, digests: torch.Tensor,
                          status: torch.Tensor, stream=None) -> None:
    D = enc_off.numel() - 1
    _check(lib().pk_digest_descriptors(ctx, _p(enc), enc.numel(), _p(enc_off), D, _p(digests), _p(status),
                                       _s(stream)), "pk_digest_descriptors")


def pk_derive_keys(ctx: int, tokens: torch.Tensor, tok_off: torch.Tensor, desc_idx: torch.Tensor,
                   digests: torch.Tensor, key_off: torch.Tensor, keys: torch.Tensor, status: torch.Tensor,
                   stream=None) -> None:
    R = tok_off.numel() - 1
    D = digests.numel() // 32
    _check(lib().pk_derive_keys(ctx, _p(tokens), tokens.numel(), _p(tok_off), R, _p(desc_idx), _p(digests), D,
                                _p(key_off), _p(keys), keys.numel() // 32, _p(status), _s(stream)),
           "pk_derive_keys")


def pk_derive_keys_enc(ctx: int, tokens: torch.Tensor, tok_off: torch.Tensor, desc_idx: torch.Tensor,
                       enc: torch.Tensor, enc_off: torch.Tensor, digests: torch.Tensor, key_off: torch.Tensor,
                       keys: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    R = tok_off.numel() - 1
    D = enc_off.numel() - 1
    _check(lib().pk_derive_keys_enc(ctx, _p(tokens), tokens.numel(), _p(tok_off), R, _p(desc_idx), _p(enc),
                                    enc.numel(), _p(enc_off), D, _p(digests), _p(key_off), _p(keys),
                                    keys.numel() // 32, _p(status), _s(stream)), "pk_derive_keys_enc")


def pk_lookup(ctx: int, keys: torch.Tensor, key_off: torch.Tensor, hit_chunks: torch.Tensor,
              slots: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    R = key_off.numel() - 1
    _check(lib().pk_lookup(ctx, _p(keys), _p(key_off), R, keys.numel() // 32, _p(hit_chunks), _p(slots),
                           _p(status), _s(stream)), "pk_lookup")


def pk_store(ctx: int, keys: torch.Tensor, slots: torch.Tensor, result: torch.Tensor, slot_out: torch.Tensor,
             status: torch.Tensor, key_off: Optional[torch.Tensor] = None,
             hit_chunks: Optional[torch.Tensor] = None, stream=None) -> None:
    n = keys.numel() // 32
    R = 0 if key_off is None else key_off.numel() - 1
    _check(lib().pk_store(ctx, _p(keys), _p(slots), n, _p(key_off), _p(hit_chunks), R, _p(result), _p(slot_out),
                          _p(status), _s(stream)), "pk_store")


def pk_lookup_store(ctx: int, keys: torch.Tensor, new_slots: torch.Tensor, key_off: torch.Tensor,
                    hit_chunks: torch.Tensor, slots: torch.Tensor, result: torch.Tensor, slot_out: torch.Tensor,
                    status: torch.Tensor, stream=None) -> None:
    R = key_off.numel() - 1
    _check(lib().pk_lookup_store(ctx, _p(keys), _p(new_slots), _p(key_off), R, keys.numel() // 32,
                                 _p(hit_chunks), _p(slots), _p(result), _p(slot_out), _p(status), _s(stream)),
           "pk_lookup_store")


def pk_derive_lookup_store(ctx: int, tokens: torch.Tensor, tok_off: torch.Tensor, desc_idx: torch.Tensor,
                           enc: torch.Tensor, enc_off: torch.Tensor, digests: torch.Tensor, key_off: torch.Tensor,
                           keys: torch.Tensor, new_slots: torch.Tensor, hit_chunks: torch.Tensor, slots: torch.Tensor,
                           result: torch.Tensor, slot_out: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    R = tok_off.numel() - 1
    D = enc_off.numel() - 1
    _check(lib().pk_derive_lookup_store(ctx, _p(tokens), tokens.numel(), _p(tok_off), R, _p(desc_idx), _p(enc),
                                        enc.numel(), _p(enc_off), D, _p(digests), _p(key_off), _p(keys),
                                        keys.numel() // 32, _p(new_slots), _p(hit_chunks), _p(slots), _p(result),
                                        _p(slot_out), _p(status), _s(stream)), "pk_derive_lookup_store")


def pk_compare_pages(slots: torch.Tensor, pages: torch.Tensor, ref_pages: torch.Tensor, verdict: torch.Tensor,
                     counts: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    """pages: uint8 [n, page_bytes]; ref_pages: uint8 [n_ref, page_bytes]; counts: int64[3] (accumulated)."""
    n, page_bytes = pages.shape
    _check(lib().pk_compare_pages(_p(slots), _p(pages), _p(ref_pages), n, ref_pages.shape[0], page_bytes,
                                  _p(verdict), _p(counts), _p(status), _s(stream)), "pk_compare_pages")


def pk_content_scratch_bytes(n_bytes: int) -> int:
    return int(lib().pk_content_scratch_bytes(n_bytes))


def pk_content_digest(data: torch.Tensor, scratch: torch.Tensor, top: torch.Tensor, stream=None) -> None:
    """top (uint8[32], device) = tree top of the bytes of `data` (a contiguous device tensor)."""
    n = data.numel() * data.element_size()
    _check(lib().pk_content_digest(_p(data), n, _p(scratch), scratch.numel(), _p(top), _s(stream)),
           "pk_content_digest")


def pk_content_scratch_bytes_batch(sizes) -> int:
    arr = (ctypes.c_uint64 * max(len(sizes), 1))(*[int(x) for x in sizes])
    return int(lib().pk_content_scratch_bytes_batch(arr, len(sizes)))


def pk_content_digests(datas, scratch: torch.Tensor, tops: torch.Tensor, stream=None) -> None:
    """tops (uint8[n, 32], device) = the tree tops of the contiguous device tensors `datas`."""
    n = len(datas)
    ptrs = (ctypes.c_void_p * max(n, 1))(*[_p(d) for d in datas])
    sizes = (ctypes.c_uint64 * max(n, 1))(*[d.numel() * d.element_size() for d in datas])
    _check(lib().pk_content_digests(ptrs, sizes, n, _p(scratch), scratch.numel(), _p(tops), _s(stream)),
           "pk_content_digests")


def _pkb(b: bytes):
    buf = ctypes.create_string_buffer(bytes(b), max(len(b), 1))
    return pk_bytes(ctypes.cast(buf, ctypes.c_void_p), len(b)), buf


def pk_tensor_identity(name, dtype, shape, n_bytes: int, top: bytes) -> bytes:
    nb, k1 = _pkb(name.encode() if isinstance(name, str) else name)
    db, k2 = _pkb(dtype.encode() if isinstance(dtype, str) else dtype)
    dims = (ctypes.c_int64 * max(len(shape), 1))(*[int(x) for x in shape])
    t = (ctypes.c_uint8 * 32).from_buffer_copy(bytes(top))
    out = (ctypes.c_uint8 * 32)()
    _check(lib().pk_tensor_identity(ctypes.byref(nb), ctypes.byref(db), dims, len(shape), n_bytes, t, out),
           "pk_tensor_identity")
    return bytes(out)


def pk_adapter_identity(tensor_ids, config) -> bytes:
    ids = np.frombuffer(b"".join(bytes(x) for x in tensor_ids), np.uint8) if tensor_ids else np.zeros(32, np.uint8)
    keep = [_pkb(c.encode() if isinstance(c, str) else c) for c in config]
    arr = (pk_bytes * max(len(keep), 1))(*[k[0] for k in keep])
    out = (ctypes.c_uint8 * 32)()
    _check(lib().pk_adapter_identity(ids.ctypes.data, len(tensor_ids), arr, len(keep), out), "pk_adapter_identity")
    return bytes(out)


def pk_stamps_bytes(capacity_log2: int) -> int:
    return int(lib().pk_stamps_bytes(capacity_log2))


def pk_attach_stamps(ctx: int, stamps: Optional[torch.Tensor], stream=None) -> None:
    """Budget mode on (stamps: device buffer of pk_stamps_bytes, zeroed here) or off (None)."""
    nbytes = 0 if stamps is None else stamps.numel() * stamps.element_size()
    _check(lib().pk_attach_stamps(ctx, _p(stamps), nbytes, _s(stream)), "pk_attach_stamps")


def pk_evict_scratch_bytes(capacity_log2: int) -> int:
    return int(lib().pk_evict_scratch_bytes(capacity_log2))


def pk_evict(ctx: int, budget: int, keep: int, scratch: torch.Tensor, evicted: Optional[torch.Tensor],
             n_evicted: Optional[torch.Tensor], status: torch.Tensor, stream=None) -> None:
    """evicted: uint32/int32 [cap] device (or None); n_evicted: int64[1] device (or None)."""
    _check(lib().pk_evict(ctx, budget, keep, _p(scratch), scratch.numel(), _p(evicted),
                          0 if evicted is None else evicted.numel(), _p(n_evicted), _p(status), _s(stream)),
           "pk_evict")


def pk_evict_barrier_timeout_test(ctx: int, budget: int, scratch: torch.Tensor, spin_limit: int,
                                  status: torch.Tensor, stream=None) -> None:
    """Test hook: pk_evict with CTA 0 withholding its first barrier arrival and
    the waits bounded at spin_limit polls (the status must end PK_ERR_TIMEOUT)."""
    _check(lib().pk_evict_barrier_timeout_test(ctx, budget, _p(scratch), scratch.numel(), spin_limit, _p(status),
                                               _s(stream)), "pk_evict_barrier_timeout_test")


def pk_key_string(key16: bytes) -> str:
    """The 22 base64 characters of a 16-byte key prefix (host)."""
    if len(bytes(key16)) != 16:
        raise PKError(PK_ERR_ARG, "pk_key_string")
    k = (ctypes.c_uint8 * 16).from_buffer_copy(bytes(key16))
    out = (ctypes.c_char * 22)()
    _check(lib().pk_key_string(k, out), "pk_key_string")
    return out.raw.decode("ascii")


def pk_model_tag(desc) -> str:
    """The 22-character hash of the model identity and worker provenance (host)."""
    d = _descs([desc]) if isinstance(desc, Mapping) else _descs(desc)
    out = (ctypes.c_char * 22)()
    _check(lib().pk_model_tag(d.array, out), "pk_model_tag")
    return out.raw.decode("ascii")


def pk_key_strings(keys: torch.Tensor, prefix: bytes, width: int, out: torch.Tensor, n: Optional[int] = None,
                   stream=None) -> None:
    """out (uint8 [n, width], device): row i = prefix || base64 of keys[i, :16] || zero fill."""
    n = keys.shape[0] if n is None else n
    pre = bytes(prefix)
    buf = ctypes.create_string_buffer(pre, max(len(pre), 1))
    _check(lib().pk_key_strings(_p(keys), n, ctypes.cast(buf, ctypes.c_void_p), len(pre), width, _p(out),
                                _s(stream)), "pk_key_strings")


def pk_table_save(ctx: int, dst: torch.Tensor, stream=None) -> None:
    """dst: host or device memory, on any device."""
    at = dst.data_ptr() if dst.numel() else None
    _check(lib().pk_table_save(ctx, at, dst.numel() * dst.element_size(), _s(stream)), "pk_table_save")


def pk_table_load(ctx: int, src: torch.Tensor, stream=None) -> None:
    _check(lib().pk_table_load(ctx, _p(src), src.numel() * src.element_size(), _s(stream)), "pk_table_load")


# -- KV pages ---------------------------------------------------------------------------------------------------------
# A decode step makes several of these calls, so their marshalling is kept short: tensors are looked at once, and texts
# of errors are made only when they are raised.
_KV_DTYPES = {torch.bfloat16: PK_BF16, torch.float16: PK_FP16}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(stream, t: torch.Tensor) -> Optional[int]:
    """Handle of `stream`, or of the current stream of t's device."""
    if stream is None and _raw_stream is not None and t.is_cuda:
        return _raw_stream(t.device.index)
    return _s(stream)


def _refuse(where: str, what: str):
    raise PKError(PK_ERR_ARG, f"{where}: {what}")


def _here(where: str, kv: Optional[pk_kv_cache] = None) -> int:
    """The current device, on which a call's kernels run and all its tensors have to be, the pool among them."""
    try:
        dev = _current_device()
    except RuntimeError:  # no GPU
        dev = -2  # no tensor's: on the host it is -1
    if kv is not None and kv.device is not None and kv.device != dev:
        _refuse(where, "the pool is on another device than the current one")
    return dev


def _ints(t: torch.Tensor, dtype, n: int, dev: int, where: str, what: str) -> Optional[int]:
    """Pointer of a contiguous array of n entries on device `dev`."""
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous() or t.get_device() != dev:
        _refuse(where, what + ", on the current device")
    return t.data_ptr() if n else None


def _heads(t: torch.Tensor, dev: int, where: str):
    """pk_heads of [tokens, heads, head_dim], or [R, n, heads, head_dim] whose first two dimensions run on as one; the
    last dimension contiguous."""
    shape, stride = t.shape, t.stride()
    if len(shape) == 4:
        a, b = stride[0], stride[1]
        if shape[0] > 1 and shape[1] > 1 and a != shape[1] * b:
            _refuse(where, "the first two dimensions do not run on as one")
        n, ts = shape[0] * shape[1], b if shape[1] > 1 else a
    elif len(shape) == 3:
        n, ts = shape[0], stride[0]
    else:
        _refuse(where, "a [tokens, heads, head_dim] tensor")
    if t.numel() == 0:
        return pk_heads(None, 0, 0)
    if (stride[-1] != 1 and shape[-1] > 1) or t.get_device() != dev:
        _refuse(where, "rows are contiguous, on the current device")
    if t.requires_grad and torch.is_grad_enabled():
        _refuse(where, "no gradient is computed: detach, or call under torch.no_grad()")
    return pk_heads(t.data_ptr(), ts if n > 1 else 0, stride[-2] if shape[-2] > 1 else 0)


def _buffer(t: Optional[torch.Tensor], dev: int, where: str) -> Optional[int]:
    """Pointer of a status word or scratch (None for None)."""
    if t is None:
        return None
    if t.get_device() != dev:
        _refuse(where, "status and scratch are on the current device")
    return t.data_ptr() if t.numel() else None


def _dtype(where: str, first: torch.Tensor, *others) -> int:
    d = first.dtype
    for t in others:
        if t.dtype is not d:
            _refuse(where, "tensors of one type")
    code = _KV_DTYPES.get(d)
    if code is None:
        _refuse(where, "16-bit tensors (bfloat16 or float16)")
    return code


def pk_kv_page_bytes(page_tokens: int, kv_heads: int, head_dim: int) -> int:
    return int(lib().pk_kv_page_bytes(page_tokens, kv_heads, head_dim))


def _kv_move(fn: str, call, kv: pk_kv_cache, k, v, tok_off, start, pages, status, stream) -> None:
    dev = _here(fn, kv)
    R = start.numel()
    shape = k.shape
    if v.shape != shape or len(shape) != 3 or shape[1] != kv.kv_heads or shape[2] != kv.head_dim:
        _refuse(fn, "k and v are [tokens, kv_heads, head_dim]")
    if pages.dim() != 2 or pages.shape[0] != R:
        _refuse(fn, "pages is [R, page_stride]")
    width = pages.shape[1]
    rc = call(ctypes.byref(kv), _dtype(fn, k, v), ctypes.byref(_heads(k, dev, fn)), ctypes.byref(_heads(v, dev, fn)), shape[0],
              _ints(tok_off, torch.int64, R + 1, dev, fn, "tok_off is contiguous int64[R+1]"),
              _ints(start, torch.int32, R, dev, fn, "start is contiguous int32[R]"), R,
              _ints(pages, torch.int32, R * width, dev, fn, "pages is contiguous int32"), width, _buffer(status, dev, fn),
              _stream_of(stream, k))
    if rc:
        _check(rc, fn)


def pk_kv_write(kv: pk_kv_cache, k: torch.Tensor, v: torch.Tensor, tok_off: torch.Tensor, start: torch.Tensor,
                pages: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    """k, v: [tokens, kv_heads, head_dim] bf16 / fp16 (strided); tok_off: int64[R+1]; start: int32[R]; pages:
    int32 [R, page_stride] holding uint32 slots."""
    _kv_move("pk_kv_write", lib().pk_kv_write, kv, k, v, tok_off, start, pages, status, stream)


def pk_kv_read(kv: pk_kv_cache, k: torch.Tensor, v: torch.Tensor, tok_off: torch.Tensor, start: torch.Tensor,
               pages: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    """k, v: outputs; the other arguments as pk_kv_write."""
    _kv_move("pk_kv_read", lib().pk_kv_read, kv, k, v, tok_off, start, pages, status, stream)


def pk_attend_prompt_scratch_bytes(R: int) -> int:
    return int(lib().pk_attend_prompt_scratch_bytes(R))


def pk_attend_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                     lse: Optional[torch.Tensor], q_off: torch.Tensor, k_off: torch.Tensor, scale: float,
                     scratch: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    """q, out: [n_q, q_heads, D]; k, v: [n_k, kv_heads, D]; q_off, k_off: int64[R+1]; lse: float32 [n_q, q_heads]."""
    fn = "pk_attend_prompt"
    dev = _here(fn)
    R = q_off.numel() - 1
    qs, ks = q.shape, k.shape
    if len(qs) != 3 or len(ks) != 3 or v.shape != ks or out.shape != qs or qs[2] != ks[2]:
        _refuse(fn, "q, out [n_q, q_heads, D], k, v [n_k, kv_heads, D]")
    if R < 0:
        _refuse(fn, "q_off is int64[R+1]")
    z = lse
    if lse is not None:
        z = _ints(lse, torch.float32, qs[0] * qs[1], dev, fn, "lse is contiguous float32 [n_q, q_heads]")
    rc = lib().pk_attend_prompt(_dtype(fn, q, k, v, out), ctypes.byref(_heads(q, dev, fn)), ctypes.byref(_heads(k, dev, fn)),
                                ctypes.byref(_heads(v, dev, fn)), ctypes.byref(_heads(out, dev, fn)), z, qs[0], ks[0],
                                _ints(q_off, torch.int64, R + 1, dev, fn, "q_off is contiguous int64[R+1]"),
                                _ints(k_off, torch.int64, R + 1, dev, fn, "k_off is contiguous int64[R+1]"), R, qs[1],
                                ks[1], qs[2], scale, _buffer(scratch, dev, fn), scratch.numel(), _buffer(status, dev, fn),
                                _stream_of(stream, q))
    if rc:
        _check(rc, fn)


def pk_attend_cache_scratch_bytes(kv: pk_kv_cache, R: int, n_q: int, q_heads: int, page_stride: int,
                                  weigh: bool) -> int:
    return int(lib().pk_attend_cache_scratch_bytes(ctypes.byref(kv), R, n_q, q_heads, page_stride, int(weigh)))


def pk_attend_cache(kv: pk_kv_cache, q: torch.Tensor, out: torch.Tensor, lse: Optional[torch.Tensor], n_q: int,
                    kv_len: torch.Tensor, pages: torch.Tensor, scale: float, page_weight: Optional[torch.Tensor],
                    scratch: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    """q, out: [R * n_q, q_heads, D] or [R, n_q, q_heads, D]; lse: float32, R * n_q * q_heads; kv_len: int32[R]; pages:
    int32 and page_weight: float32 [R, page_stride]."""
    fn = "pk_attend_cache"
    dev = _here(fn, kv)
    R = kv_len.numel()
    qs = q.shape
    if out.shape != qs or len(qs) not in (3, 4) or q.numel() != R * n_q * qs[-2] * qs[-1] or qs[-1] != kv.head_dim:
        _refuse(fn, "q, out are [R * n_q, q_heads, head_dim]")
    if pages.dim() != 2 or pages.shape[0] != R:
        _refuse(fn, "pages is [R, page_stride]")
    width = pages.shape[1]
    z = w = None
    if lse is not None:
        z = _ints(lse, torch.float32, R * n_q * qs[-2], dev, fn, "lse is contiguous float32, R * n_q * q_heads")
    if page_weight is not None:
        if page_weight.shape != pages.shape:
            _refuse(fn, "page_weight is [R, page_stride]")
        w = _ints(page_weight, torch.float32, R * width, dev, fn, "page_weight is contiguous float32")
    rc = lib().pk_attend_cache(ctypes.byref(kv), _dtype(fn, q, out), ctypes.byref(_heads(q, dev, fn)),
                               ctypes.byref(_heads(out, dev, fn)), z, R, n_q, qs[-2], scale,
                               _ints(kv_len, torch.int32, R, dev, fn, "kv_len is contiguous int32[R]"),
                               _ints(pages, torch.int32, R * width, dev, fn, "pages is contiguous int32"), width, w,
                               _buffer(scratch, dev, fn), scratch.numel(), _buffer(status, dev, fn),
                                _stream_of(stream, q))
    if rc:
        _check(rc, fn)


def pk_evict_pages(pages: torch.Tensor, weight: torch.Tensor, kv_len: torch.Tensor, page_tokens: int, budget: int,
                   sinks: int, recent: int, pages_out: torch.Tensor, weight_out: torch.Tensor,
                   kv_len_out: torch.Tensor, evicted: Optional[torch.Tensor], status: torch.Tensor,
                   stream=None) -> None:
    """pages: int32 and weight: float32 [R, page_stride]; kv_len, kv_len_out: int32[R]; pages_out: int32 and
    weight_out: float32 [R, budget]; evicted: int32 [R, page_stride] or None."""
    fn = "pk_evict_pages"
    dev = _here(fn)
    R = kv_len.numel()
    if pages.dim() != 2 or pages.shape[0] != R or weight.shape != pages.shape:
        _refuse(fn, "pages, weight are [R, page_stride]")
    if page_tokens < 0 or budget < 0 or sinks < 0 or recent < 0:
        _refuse(fn, "counts are not negative")
    width = pages.shape[1]
    n = R * width
    rc = lib().pk_evict_pages(_ints(pages, torch.int32, n, dev, fn, "pages is contiguous int32"),
                              _ints(weight, torch.float32, n, dev, fn, "weight is contiguous float32"),
                              _ints(kv_len, torch.int32, R, dev, fn, "kv_len is contiguous int32[R]"), R, width,
                              page_tokens, budget, sinks, recent,
                              _ints(pages_out, torch.int32, R * budget, dev, fn, "pages_out is int32[R, budget]"),
                              _ints(weight_out, torch.float32, R * budget, dev, fn, "weight_out is float32[R, budget]"),
                              _ints(kv_len_out, torch.int32, R, dev, fn, "kv_len_out is int32[R]"),
                              None if evicted is None else
                              _ints(evicted, torch.int32, n, dev, fn, "evicted is int32[R, page_stride]"),
                              _buffer(status, dev, fn), _stream_of(stream, pages))
    if rc:
        _check(rc, fn)


def pk_store_noalloc(table: torch.Tensor, capacity_log2: int, keys: torch.Tensor, slots: torch.Tensor,
                     result: torch.Tensor, slot_out: torch.Tensor, status: torch.Tensor, max_probe: int = 0,
                     key_off: Optional[torch.Tensor] = None, hit_chunks: Optional[torch.Tensor] = None,
                     stream=None) -> None:
    """pk_store without a context, for callers that cannot allocate device
    memory; the table tensor must be zero-filled before its first use."""
    cfg = pk_config(1, capacity_log2, max_probe, _p(table), table.numel() * table.element_size())
    n = keys.numel() // 32
    R = 0 if key_off is None else key_off.numel() - 1
    _check(lib().pk_store_noalloc(ctypes.byref(cfg), _p(keys), _p(slots), n, _p(key_off), _p(hit_chunks), R,
                                  _p(result), _p(slot_out), _p(status), _s(stream)), "pk_store_noalloc")


def pk_entries(ctx: int, stream=None) -> int:
    v = ctypes.c_uint64(0)
    _check(lib().pk_entries(ctx, ctypes.byref(v), _s(stream)), "pk_entries")
    return int(v.value)
