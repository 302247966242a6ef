"""Python binding of libkvq.so (ctypes): same names as the C ABI in include/kvq.h.

Argument marshalling only.  Tensors are passed by their device pointers and
the current HIP stream of torch; every step of the computation runs in the
library's kernels.  There is no fallback: without the built library every
call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkvq.so")

OK, ERR_ARG, ERR_UNSUPPORTED, ERR_CAPACITY, ERR_RANGE, ERR_STATE, ERR_HIP = range(7)
STATUS_NAMES = ["KVQ_OK", "KVQ_ERR_ARG", "KVQ_ERR_UNSUPPORTED", "KVQ_ERR_CAPACITY",
                "KVQ_ERR_RANGE", "KVQ_ERR_STATE", "KVQ_ERR_HIP"]

EXPORTED = ["kvq_cache_bytes", "kvq_cache_init", "kvq_cache_destroy", "kvq_cache_reset",
            "kvq_seq_len", "kvq_seq_release", "kvq_free_pages",
            "kvq_append", "kvq_workspace_bytes", "kvq_decode_attention", "kvq_decode_attention_noalloc",
            "kvq_append_decode",
            "kvq_decode_partials", "kvq_decode_merge", "kvq_chunk_workspace_bytes", "kvq_chunk_attention",
            "kvq_window_workspace_bytes", "kvq_window_attention",
            "kvq_dequant", "kvq_export_bytes", "kvq_export", "kvq_check",
            "kvq_set_split_tokens", "kvq_last_error", "kvq_version",
            "kvq_read_probe", "kvq_read_probe_sink_bytes",
            "dgap_workspace_bytes", "dgap_info_floats", "dgap_restore",
            "dgap_sample_workspace_bytes", "dgap_sample",
            "dgap_distill_workspace_bytes", "dgap_distill", "dgap_distill_backward"]


class KvqError(RuntimeError):
    def __init__(self, status: int, message: str):
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__(f"{name}: {message}")
        self.status = status


class CacheDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_tokens", ctypes.c_int32), ("key_group", ctypes.c_int32),
                ("value_group", ctypes.c_int32), ("fp16_window", ctypes.c_int32),
                ("bits_k", ctypes.POINTER(ctypes.c_uint8)), ("bits_v", ctypes.POINTER(ctypes.c_uint8)),
                ("page_tokens", ctypes.c_int32), ("num_pages", ctypes.c_int32)]


class DgapParams(ctypes.Structure):
    """dgap_params of include/dgap.h (weights are device pointers)."""
    _fields_ = [("vocab", ctypes.c_int32), ("k", ctypes.c_int32), ("hidden_det", ctypes.c_int32),
                ("hidden_corr", ctypes.c_int32), ("tau", ctypes.c_float), ("det_b2", ctypes.c_float),
                ("corr_b2", ctypes.c_float), ("pad", ctypes.c_int32),
                ("det_w1", ctypes.c_void_p), ("det_b1", ctypes.c_void_p), ("det_w2", ctypes.c_void_p),
                ("corr_w1", ctypes.c_void_p), ("corr_b1", ctypes.c_void_p), ("corr_w2", ctypes.c_void_p)]


class DgapSampling(ctypes.Structure):
    """dgap_sampling of include/dgap.h (device pointers)."""
    _fields_ = [("logits", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("type", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("vocab", ctypes.c_int32), ("pad", ctypes.c_int32),
                ("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
                ("min_p", ctypes.c_void_p), ("uniform", ctypes.c_void_p)]


class DgapDistillation(ctypes.Structure):
    """dgap_distillation of include/dgap.h (device pointers)."""
    _fields_ = [("logits", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("type", ctypes.c_int32),
                ("rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("k", ctypes.c_int32),
                ("teacher", ctypes.c_void_p), ("index", ctypes.c_void_p), ("temperature", ctypes.c_float),
                ("pad", ctypes.c_int32)]


_lib = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with paper_2607_16248_amd/build.py "
                          "(the HIP library has no fallback)")
    L = ctypes.CDLL(LIB_PATH)
    P, S, I32, I64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64
    D = ctypes.POINTER(CacheDesc)
    sig = {
        "kvq_cache_bytes": ([D], S),
        "kvq_cache_init": ([ctypes.POINTER(P), D, P, S], ctypes.c_int),
        "kvq_cache_destroy": ([P], None),
        "kvq_cache_reset": ([P, P], ctypes.c_int),
        "kvq_seq_len": ([P, I32], I64),
        "kvq_seq_release": ([P, I32], ctypes.c_int),
        "kvq_free_pages": ([P], I64),
        "kvq_append": ([P, P, P, I32, ctypes.POINTER(I32), P], ctypes.c_int),
        "kvq_workspace_bytes": ([P], S),
        "kvq_decode_attention": ([P, P, P, P, S, P], ctypes.c_int),
        "kvq_decode_attention_noalloc": ([P, P, P, P], ctypes.c_int),
        "kvq_chunk_workspace_bytes": ([P, ctypes.c_int32], S),
        "kvq_chunk_attention": ([P, P, ctypes.c_int32, P, P, S, P], ctypes.c_int),
        "kvq_window_workspace_bytes": ([P, I32, I32, I32], S),
        "kvq_window_attention": ([P, P, I32, I32, I32, P, P, S, P], ctypes.c_int),
        "kvq_append_decode": ([P, P, P, I32, ctypes.POINTER(I32), P, P, P, S, P], ctypes.c_int),
        "kvq_decode_partials": ([P, P, P, S, P], ctypes.c_int),
        "kvq_decode_merge": ([P, P, P, P], ctypes.c_int),
        "kvq_dequant": ([P, I32, I32, I32, P, P, P], ctypes.c_int),
        "kvq_export_bytes": ([P, I32, I32], S),
        "kvq_export": ([P, I32, I32, P, S, P], ctypes.c_int),
        "kvq_check": ([P, P], ctypes.c_int),
        "kvq_set_split_tokens": ([P, I32], ctypes.c_int),
        "kvq_last_error": ([], ctypes.c_char_p),
        "kvq_version": ([], ctypes.c_char_p),
        "kvq_read_probe": ([P, S, P, P], ctypes.c_int),
        "kvq_read_probe_sink_bytes": ([], S),
        "dgap_workspace_bytes": ([I32, I32, I32], S),
        "dgap_info_floats": ([I32], S),
        "dgap_restore": ([ctypes.POINTER(DgapParams), P, I32, P, S, P, P], ctypes.c_int),
        "dgap_sample_workspace_bytes": ([I32, I32], S),
        "dgap_distill_workspace_bytes": ([I32, I32], S),
        "dgap_distill": ([ctypes.POINTER(DgapDistillation), P, P, P, I64, P, P, S, P], ctypes.c_int),
        "dgap_distill_backward": ([ctypes.POINTER(DgapDistillation), P, P, P, I64, P], ctypes.c_int),
        "dgap_sample": ([ctypes.POINTER(DgapSampling), P, P, P, S, P], ctypes.c_int),
    }
    for name, (args, res) in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = res
    _lib = L
    return L


def _check(status: int):
    if status != OK:
        raise KvqError(status, kvq_last_error())


def _ptr(x) -> Optional[int]:
    """Device address of a tensor, or an int address, or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        if not torch.cuda.is_available():
            return None
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_desc(batch: int, num_q_heads: int, num_kv_heads: int, head_dim: int, max_tokens: int,
              key_group: int, value_group: int, fp16_window: int, bits_k: Sequence[int],
              bits_v: Sequence[int], page_tokens: int = 0, num_pages: int = 0):
    """A descriptor plus the host arrays it points to (keep both alive)."""
    bk = (ctypes.c_uint8 * max(1, len(bits_k)))(*bits_k)
    bv = (ctypes.c_uint8 * max(1, len(bits_v)))(*bits_v)
    d = CacheDesc(batch, num_q_heads, num_kv_heads, head_dim, max_tokens, key_group, value_group,
                  fp16_window, ctypes.cast(bk, ctypes.POINTER(ctypes.c_uint8)),
                  ctypes.cast(bv, ctypes.POINTER(ctypes.c_uint8)), page_tokens, num_pages)
    d._keep = (bk, bv)
    return d


def kvq_cache_bytes(desc: CacheDesc) -> int:
    return int(lib().kvq_cache_bytes(ctypes.byref(desc)))


def kvq_cache_init(desc: CacheDesc, arena, arena_bytes: Optional[int] = None) -> int:
    """Handle (an int) over ``arena`` (a device tensor or address)."""
    if arena_bytes is None:
        arena_bytes = arena.numel() * arena.element_size()
    h = ctypes.c_void_p()
    _check(lib().kvq_cache_init(ctypes.byref(h), ctypes.byref(desc), _ptr(arena), int(arena_bytes)))
    return h.value


def kvq_cache_destroy(cache: int) -> None:
    lib().kvq_cache_destroy(cache)


def kvq_cache_reset(cache: int, stream=None) -> None:
    _check(lib().kvq_cache_reset(cache, _stream(stream)))


def kvq_seq_len(cache: int, seq: int) -> int:
    return int(lib().kvq_seq_len(cache, seq))


def kvq_seq_release(cache: int, seq: int) -> None:
    _check(lib().kvq_seq_release(cache, seq))


def kvq_free_pages(cache: int) -> int:
    return int(lib().kvq_free_pages(cache))


def kvq_append(cache: int, K, V, n_new: Sequence[int], n_max: Optional[int] = None, stream=None) -> None:
    """K, V: fp16 [batch][n_max][Hkv][d] on the device; n_new: per-sequence counts."""
    n = (ctypes.c_int32 * max(1, len(n_new)))(*n_new)
    if n_max is None:
        n_max = int(K.shape[1]) if K is not None and not isinstance(K, int) else max(n_new, default=0)
    _check(lib().kvq_append(cache, _ptr(K), _ptr(V), int(n_max), n, _stream(stream)))


def kvq_workspace_bytes(cache: int) -> int:
    return int(lib().kvq_workspace_bytes(cache))


def kvq_decode_attention(cache: int, q, out, ws, ws_bytes: Optional[int] = None, stream=None) -> None:
    """q: fp16 [batch][Hq][d]; out: fp32 [batch][Hq][d]; ws: scratch bytes."""
    if ws_bytes is None:
        ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().kvq_decode_attention(cache, _ptr(q), _ptr(out), _ptr(ws), int(ws_bytes), _stream(stream)))


def kvq_decode_attention_noalloc(cache: int, q, out, stream=None) -> None:
    """kvq_decode_attention with the library's own scratch array as workspace."""
    _check(lib().kvq_decode_attention_noalloc(cache, _ptr(q), _ptr(out), _stream(stream)))


def kvq_chunk_workspace_bytes(cache: int, n_q: int) -> int:
    return int(lib().kvq_chunk_workspace_bytes(cache, int(n_q)))


def kvq_chunk_attention(cache: int, q, n_q: int, out, ws, ws_bytes: Optional[int] = None, stream=None) -> None:
    """The last n_q tokens of every sequence attend causally: q fp16 [batch][n_q][Hq][d],
    out fp32 [batch][n_q][Hq][d]."""
    if ws_bytes is None:
        ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().kvq_chunk_attention(cache, _ptr(q), int(n_q), _ptr(out), _ptr(ws), int(ws_bytes),
                                     _stream(stream)))


_I32 = 1 << 31


def _window_sizes(n_q, window, sinks):
    """The sizes as the C interface takes them (ctypes would keep the lowest 32 bits of larger ones)."""
    if not (-_I32 <= n_q < _I32 and -_I32 <= window < _I32 and -_I32 <= sinks < _I32):
        raise ValueError(f"n_q = {n_q}, window = {window}, sinks = {sinks}: 32 bits each")
    return int(n_q), int(window), int(sinks)


def kvq_window_workspace_bytes(cache: int, n_q: int, window: int, sinks: int = 0) -> int:
    return int(lib().kvq_window_workspace_bytes(cache, *_window_sizes(n_q, window, sinks)))


def _on_device(stream, call, *tensors) -> None:
    """call(stream) on the tensors' device: one of them all, which need not be the current one."""
    device = None
    for x in tensors:
        if x is None or isinstance(x, int):
            continue
        at = x.get_device()
        if at < 0:
            raise ValueError("tensors must be on a GPU")
        if device is not None and at != device:
            raise ValueError("tensors are on different devices")
        device = at
    if device is None:  # (addresses only)
        return call(_stream(stream))
    import torch
    if stream is None:
        stream = torch.cuda.current_stream(device)
    if device == torch.cuda.current_device():
        return call(_stream(stream))
    with torch.cuda.device(device):
        call(_stream(stream))


def kvq_window_attention(cache: int, q, n_q: int, window: int, sinks: int, out, ws, ws_bytes: Optional[int] = None,
                         stream=None) -> None:
    """The last n_q tokens of every sequence attend over the last ``window`` tokens up to their own and the first
    ``sinks`` ones: q fp16 [batch][n_q][Hq][d], out fp32 [batch][n_q][Hq][d]."""
    if ws_bytes is None:
        ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    sizes = _window_sizes(n_q, window, sinks)
    _on_device(stream, lambda st: _check(lib().kvq_window_attention(
        cache, _ptr(q), *sizes, _ptr(out), _ptr(ws), int(ws_bytes), st)), q, out, ws)


def kvq_append_decode(cache: int, K, V, n_new: Sequence[int], q, out, ws, ws_bytes: Optional[int] = None,
                      n_max: Optional[int] = None, stream=None) -> None:
    """kvq_append then kvq_decode_attention in one call (two launches when no key group fills)."""
    n = (ctypes.c_int32 * max(1, len(n_new)))(*n_new)
    if n_max is None:
        n_max = int(K.shape[1]) if K is not None and not isinstance(K, int) else max(n_new, default=0)
    if ws_bytes is None:
        ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().kvq_append_decode(cache, _ptr(K), _ptr(V), int(n_max), n, _ptr(q), _ptr(out), _ptr(ws),
                                   int(ws_bytes), _stream(stream)))


def kvq_decode_partials(cache: int, q, ws, ws_bytes: Optional[int] = None, stream=None) -> None:
    """Phase 1 of decode: per-split softmax records into ``ws``."""
    if ws_bytes is None:
        ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().kvq_decode_partials(cache, _ptr(q), _ptr(ws), int(ws_bytes), _stream(stream)))


def kvq_read_probe(src, nbytes: int, sink, stream=None) -> None:
    """Diagnostics: read ``nbytes`` of the device buffer ``src`` once (streaming-read rate)."""
    _check(lib().kvq_read_probe(_ptr(src), int(nbytes), _ptr(sink), _stream(stream)))


def kvq_read_probe_sink_bytes() -> int:
    return int(lib().kvq_read_probe_sink_bytes())


def kvq_decode_merge(cache: int, ws, out, stream=None) -> None:
    """Phase 2 of decode: merge the records of ``ws`` into ``out``."""
    _check(lib().kvq_decode_merge(cache, _ptr(ws), _ptr(out), _stream(stream)))


def kvq_dequant(cache: int, seq: int, tok0: int, ntok: int, K_out, V_out, stream=None) -> None:
    _check(lib().kvq_dequant(cache, seq, tok0, ntok, _ptr(K_out), _ptr(V_out), _stream(stream)))


def kvq_export_bytes(cache: int, seq: int, kv_head: int) -> int:
    return int(lib().kvq_export_bytes(cache, seq, kv_head))


def kvq_export(cache: int, seq: int, kv_head: int, dst, nbytes: Optional[int] = None, stream=None) -> None:
    if nbytes is None:
        nbytes = dst.numel() * dst.element_size()
    _check(lib().kvq_export(cache, seq, kv_head, _ptr(dst), int(nbytes), _stream(stream)))


def kvq_check(cache: int, stream=None) -> None:
    _check(lib().kvq_check(cache, _stream(stream)))


def kvq_set_split_tokens(cache: int, tokens: int) -> None:
    _check(lib().kvq_set_split_tokens(cache, int(tokens)))


def kvq_last_error() -> str:
    return lib().kvq_last_error().decode()


def kvq_version() -> str:
    return lib().kvq_version().decode()


class KVCache:
    """A cache over a torch-allocated, zero-filled device arena."""

    def __init__(self, batch, num_q_heads, num_kv_heads, max_tokens, bits_k, bits_v,
                 key_group=32, value_group=32, fp16_window=0, head_dim=128, device="cuda",
                 page_tokens=0, num_pages=0):
        import torch
        bits_k = list(bits_k) if hasattr(bits_k, "__len__") else [bits_k] * batch
        bits_v = list(bits_v) if hasattr(bits_v, "__len__") else [bits_v] * batch
        self.desc = make_desc(batch, num_q_heads, num_kv_heads, head_dim, max_tokens, key_group,
                              value_group, fp16_window, bits_k, bits_v, page_tokens, num_pages)
        self.page_tokens, self.num_pages = page_tokens, num_pages
        self.batch, self.num_q_heads, self.num_kv_heads = batch, num_q_heads, num_kv_heads
        self.head_dim, self.key_group, self.value_group = head_dim, key_group, value_group
        self.fp16_window, self.bits_k, self.bits_v, self.max_tokens = fp16_window, bits_k, bits_v, max_tokens
        nbytes = kvq_cache_bytes(self.desc)
        if nbytes == 0:
            # surface the descriptor error through init
            kvq_cache_init(self.desc, 256, 0)
        self.arena = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        self.handle = kvq_cache_init(self.desc, self.arena)
        self.ws = self.ws_stream = None

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            try:
                kvq_cache_destroy(h)
            except TypeError:  # interpreter shutdown: module globals are already torn down
                pass
            self.handle = None

    def append(self, K, V, n_new=None, stream=None):
        if n_new is None:
            n_new = [int(K.shape[1])] * self.batch
        kvq_append(self.handle, K, V, n_new, stream=stream)

    def workspace(self):
        import torch
        need = kvq_workspace_bytes(self.handle)
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.arena.device)
            self.ws_stream = _stream(None)
        return self.ws

    def _buffers(self, stream, device, shape, out, ws_bytes):
        """``out`` (made if None) and a workspace of a call on ``stream``, made on that stream: torch's allocator gives
        a freed tensor's memory to the next tensor of the stream that it was made on, so a workspace of another stream
        than its kernels' would be somebody else's while they still write it."""
        import torch
        at = self.arena.device
        if stream is None or not torch.cuda.is_available():
            if out is None:
                out = torch.empty(shape, dtype=torch.float32, device=device)
            return out, torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device=at)
        caller = torch.cuda.current_stream(at)
        if isinstance(stream, int):  # (0, the default stream, is not a handle to torch)
            stream = torch.cuda.ExternalStream(stream, device=at) if stream else torch.cuda.default_stream(at)
        with torch.cuda.stream(stream):
            made = self._buffers(None, device, shape, out, ws_bytes)
        if out is None and made[0].is_cuda:  # (the caller may drop it with work of their own stream still to come)
            made[0].record_stream(caller)
        return made

    def _decode_buffers(self, stream, q, out):
        """``out`` (made if None), a workspace of a decode step and the call's stream: the cache's own workspace on the
        stream that it was made on, else one of the call's stream (two steps at once would write their records into
        the same one)."""
        import torch
        shape, at = (self.batch, self.num_q_heads, self.head_dim), _stream(stream)
        current = stream is None or at == _stream(None)
        if current and self.ws is None:
            self.workspace()
        if not current or at != self.ws_stream:
            return *self._buffers(stream, q.device, shape, out, kvq_workspace_bytes(self.handle)), at
        if out is None:
            out = torch.empty(shape, dtype=torch.float32, device=q.device)
        return out, self.workspace(), at

    def decode(self, q, out=None, stream=None):
        out, ws, at = self._decode_buffers(stream, q, out)
        kvq_decode_attention(self.handle, q, out, ws, stream=at)
        return out

    def chunk(self, q, out=None, stream=None):
        """Causal attention of the last q.shape[1] tokens of every sequence."""
        n_q = int(q.shape[1])
        shape = (self.batch, n_q, self.num_q_heads, self.head_dim)
        out, ws = self._buffers(stream, q.device, shape, out, kvq_chunk_workspace_bytes(self.handle, n_q))
        kvq_chunk_attention(self.handle, q, n_q, out, ws, stream=stream)
        return out

    def window(self, q, window, sinks=0, out=None, stream=None):
        """Attention of the last q.shape[1] tokens over a sliding window and the first ``sinks`` tokens."""
        import torch
        shape = (self.batch, q.shape[1], self.num_q_heads, self.head_dim)
        if q.dtype != torch.float16 or q.shape != shape or not q.is_contiguous():
            raise ValueError(f"q must be a contiguous float16 tensor of shape {shape}")
        n_q = int(q.shape[1])
        if out is not None and (out.dtype != torch.float32 or out.shape != shape or not out.is_contiguous()):
            raise ValueError(f"out must be a contiguous float32 tensor of shape {shape}")
        size = max(kvq_window_workspace_bytes(self.handle, n_q, window, sinks), 256)
        if stream is not None:
            out, ws = self._buffers(stream, q.device, shape, out, size)
        else:
            if out is None:
                out = torch.empty(shape, dtype=torch.float32, device=q.device)
            ws = torch.empty(size, dtype=torch.uint8, device=self.arena.device)
        kvq_window_attention(self.handle, q, n_q, window, sinks, out, ws, size, stream=stream)
        return out

    def append_decode(self, K, V, q, n_new=None, out=None, stream=None):
        if n_new is None:
            n_new = [int(K.shape[1])] * self.batch
        out, ws, at = self._decode_buffers(stream, q, out)
        kvq_append_decode(self.handle, K, V, n_new, q, out, ws, stream=at)
        return out

    def seq_len(self, seq):
        return kvq_seq_len(self.handle, seq)

    def release(self, seq):
        kvq_seq_release(self.handle, seq)

    def free_pages(self):
        return kvq_free_pages(self.handle)

    def export(self, seq, kv_head):
        import torch
        n = kvq_export_bytes(self.handle, seq, kv_head)
        dst = torch.zeros(max(n, 1), dtype=torch.uint8, device=self.arena.device)
        kvq_export(self.handle, seq, kv_head, dst, n)
        torch.cuda.synchronize()
        return dst[:n].cpu().numpy()

    def dequant(self, seq, tok0, ntok):
        import torch
        Ko = torch.empty((max(ntok, 1), self.num_kv_heads, self.head_dim), dtype=torch.float32,
                         device=self.arena.device)
        Vo = torch.empty_like(Ko)
        kvq_dequant(self.handle, seq, tok0, ntok, Ko, Vo)
        return Ko[:ntok], Vo[:ntok]

    def check(self):
        kvq_check(self.handle)

    def reset(self):
        kvq_cache_reset(self.handle)


# ------------------------------------------------------------------ DGAP

def dgap_workspace_bytes(batch: int, vocab: int, k: int) -> int:
    return int(lib().dgap_workspace_bytes(batch, vocab, k))


def dgap_info_floats(k: int) -> int:
    return int(lib().dgap_info_floats(k))


def dgap_params(vocab: int, k: int, tau: float, det_w1, det_b1, det_w2, det_b2: float,
                corr_w1, corr_b1, corr_w2, corr_b2: float) -> DgapParams:
    """Params from device fp32 tensors (det_w1 [12][hd], corr_w1 [17][hc], ...)."""
    return DgapParams(int(vocab), int(k), int(det_b1.numel()) if det_b1 is not None else 0,
                      int(corr_b1.numel()) if corr_b1 is not None else 0, float(tau), float(det_b2),
                      float(corr_b2), 0, _ptr(det_w1), _ptr(det_b1), _ptr(det_w2), _ptr(corr_w1),
                      _ptr(corr_b1), _ptr(corr_w2))


def dgap_restore(params: DgapParams, logits, batch: int, ws, ws_bytes: Optional[int] = None, info=None,
                 stream=None) -> None:
    """One DGAP step on ``batch`` rows of device fp32 logits, in place."""
    if ws_bytes is None:
        ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().dgap_restore(ctypes.byref(params), _ptr(logits), int(batch), _ptr(ws), int(ws_bytes),
                              _ptr(info), _stream(stream)))


# ---------------------------------- rows of logits: tokens, teacher loss

def _rows(logits):
    """(dgap_type, row stride) of a [rows][vocab] tensor whose rows are contiguous."""
    name = str(logits.dtype)
    if name not in _DGAP_TYPES:
        raise TypeError(f"logits of {name}: float32, float16 or bfloat16 are supported")
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [rows][vocab] with contiguous rows")
    return _DGAP_TYPES[name], int(logits.stride(0)) if logits.shape[0] > 1 else int(logits.shape[1])


_DGAP_TYPES = {"torch.float32": 0, "torch.float16": 1, "torch.bfloat16": 2}


def _per_row(name, x, rows, dtype):
    """A device array of one value per row, or None; its address."""
    if x is None:
        return None
    if str(x.dtype) != dtype or x.numel() != rows or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {rows} values")
    return x.data_ptr()


def dgap_sample_workspace_bytes(batch: int, vocab: int) -> int:
    return int(lib().dgap_sample_workspace_bytes(int(batch), int(vocab)))


def dgap_sample(logits, uniform, tokens, ws, temperature=None, top_k=None, top_p=None, min_p=None, logprobs=None,
                ws_bytes: Optional[int] = None, stream=None) -> None:
    """The next token of every row of ``logits`` ([rows][vocab], fp32, fp16 or bf16) from one number in [0, 1) per row.

    ``tokens`` int32 [rows] and ``logprobs`` fp32 [rows] receive the result; the settings are tensors of one value per
    row (top_k int32, the others fp32) or None.
    """
    kind, stride = _rows(logits)
    n, f32, i32 = int(logits.shape[0]), "torch.float32", "torch.int32"
    p = DgapSampling(_ptr(logits), stride, kind, n, int(logits.shape[1]), 0,
                     _per_row("temperature", temperature, n, f32), _per_row("top_k", top_k, n, i32),
                     _per_row("top_p", top_p, n, f32), _per_row("min_p", min_p, n, f32),
                     _per_row("uniform", uniform, n, f32))
    if ws_bytes is None:
        ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    out = _per_row("tokens", tokens, n, i32), _per_row("logprobs", logprobs, n, f32)
    _on_device(stream, lambda st: _check(lib().dgap_sample(ctypes.byref(p), *out, _ptr(ws), int(ws_bytes), st)),
               logits, uniform, tokens, ws, temperature, top_k, top_p, min_p, logprobs)


def dgap_distill_workspace_bytes(rows: int, vocab: int) -> int:
    return int(lib().dgap_distill_workspace_bytes(int(rows), int(vocab)))


def _distillation(logits, teacher, index, temperature, grad):
    kind, stride = _rows(logits)
    n, v, k = int(logits.shape[0]), int(logits.shape[1]), int(teacher.shape[-1])
    p = DgapDistillation(_ptr(logits), stride, kind, n, v, k, _per_row("teacher", teacher, n * k, "torch.float32"),
                         _per_row("index", index, n * k, "torch.int32"), float(temperature), 0)
    grad_stride = 0
    if grad is not None:
        if grad.dtype != logits.dtype or grad.shape != logits.shape:
            raise ValueError("grad must have the logits' type and shape")
        grad_stride = _rows(grad)[1]
    return p, grad_stride


def dgap_distill(logits, teacher, index, temperature: float, loss, ws, lse=None, grad=None, grad_loss=None,
                 ws_bytes: Optional[int] = None, stream=None) -> None:
    """The loss of every row of ``logits`` ([rows][vocab]) against a teacher's top logits, and its gradient.

    ``teacher`` fp32 and ``index`` int32 [rows][k]; ``loss``, ``lse`` and ``grad_loss`` fp32 [rows]; ``grad`` like
    ``logits`` (or ``logits`` itself), None for the loss alone.
    """
    p, grad_stride = _distillation(logits, teacher, index, temperature, grad)
    n, f32 = p.rows, "torch.float32"
    if ws_bytes is None:
        ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    out = _per_row("loss", loss, n, f32), _per_row("lse", lse, n, f32), _ptr(grad), grad_stride
    scale = _per_row("grad_loss", grad_loss, n, f32)
    _on_device(stream, lambda st: _check(lib().dgap_distill(ctypes.byref(p), *out, scale, _ptr(ws), int(ws_bytes), st)),
               logits, teacher, index, loss, ws, lse, grad, grad_loss)


def dgap_distill_backward(logits, teacher, index, temperature: float, lse, grad, grad_loss=None, stream=None) -> None:
    """The gradient alone, from the ``lse`` that dgap_distill wrote for these logits."""
    p, grad_stride = _distillation(logits, teacher, index, temperature, grad)
    n, f32 = p.rows, "torch.float32"
    args = _per_row("lse", lse, n, f32), _per_row("grad_loss", grad_loss, n, f32), _ptr(grad), grad_stride
    _on_device(stream, lambda st: _check(lib().dgap_distill_backward(ctypes.byref(p), *args, st)),
               logits, teacher, index, lse, grad, grad_loss)
