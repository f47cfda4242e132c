"""ctypes binding of include/hyp_attn.h: attention over caches that requests share and that stay within a budget.

Same names as the C ABI, argument marshalling only; PyTorch owns the memory and the streams.  Work is
enqueued on `stream` (default: torch's current one), and so is the allocation of what a call returns.
An AttnCache describes tensors that the caller goes on owning and changing: new keys are written into
k / v and counted in lens by the caller, and the next call sees them.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional, Tuple

import torch

from .binding import HYP_BF16, HYP_F32, HYP_OK, HypError, load_library

EXPORTS_ATTN = ("attn_workspace_bytes", "attn_prompt", "attn_token", "attn_received", "attn_evict_workspace_bytes", "attn_evict",
                "attn_last_error")


class _Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p),
                ("k_page_stride", C.c_int64), ("k_head_stride", C.c_int64), ("k_key_stride", C.c_int64),
                ("v_page_stride", C.c_int64), ("v_head_stride", C.c_int64), ("v_key_stride", C.c_int64),
                ("page_table", C.c_void_p), ("pages_per_request", C.c_int32), ("page_keys", C.c_int32), ("n_pages", C.c_int32),
                ("lens", C.c_void_p), ("most", C.c_int32),
                ("n_requests", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("prefix_k", C.c_void_p), ("prefix_v", C.c_void_p),
                ("prefix_k_head_stride", C.c_int64), ("prefix_k_key_stride", C.c_int64),
                ("prefix_v_head_stride", C.c_int64), ("prefix_v_key_stride", C.c_int64), ("prefix_len", C.c_int32),
                ("key_pos", C.c_void_p), ("key_doc", C.c_void_p),
                ("key_pos_request_stride", C.c_int64), ("key_pos_head_stride", C.c_int64),
                ("key_doc_request_stride", C.c_int64), ("key_doc_head_stride", C.c_int64)]


class _Rule(C.Structure):
    _fields_ = [("scale", C.c_float), ("cap", C.c_float), ("slopes", C.c_void_p)]


class _Rows(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_row_stride", C.c_int64), ("q_head_stride", C.c_int64), ("n_rows", C.c_int64), ("n_q_heads", C.c_int32),
                ("q_start", C.c_void_p), ("see_all", C.c_void_p), ("q_pos", C.c_void_p), ("q_doc", C.c_void_p)]


class _Out(C.Structure):
    _fields_ = [("out", C.c_void_p), ("out_row_stride", C.c_int64), ("out_head_stride", C.c_int64), ("lse", C.c_void_p)]


class _Totals(C.Structure):
    _fields_ = [("in_", C.c_void_p), ("out", C.c_void_p), ("in_request_stride", C.c_int64), ("in_head_stride", C.c_int64),
                ("out_request_stride", C.c_int64), ("out_head_stride", C.c_int64)]


_READY = None


def _lib() -> C.CDLL:
    global _READY
    if _READY is None:
        lib = load_library()
        cache, rule, rows, out, totals = (C.POINTER(t) for t in (_Cache, _Rule, _Rows, _Out, _Totals))
        lib.attn_workspace_bytes.restype = C.c_size_t
        lib.attn_workspace_bytes.argtypes = [cache, rows, totals]
        lib.attn_prompt.restype = C.c_int
        lib.attn_prompt.argtypes = [cache, rule, rows, out, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.attn_token.restype = C.c_int
        lib.attn_token.argtypes = [cache, rule, rows, out, totals, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.attn_received.restype = C.c_int
        lib.attn_received.argtypes = [cache, rule, rows, C.c_void_p, C.c_int32, totals, C.c_void_p]
        lib.attn_evict_workspace_bytes.restype = C.c_size_t
        lib.attn_evict_workspace_bytes.argtypes = [cache, C.c_int32]
        lib.attn_evict.restype = C.c_int
        lib.attn_evict.argtypes = [cache, cache, totals, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.attn_last_error.restype = C.c_char_p
        lib.attn_last_error.argtypes = []
        _READY = lib
    return _READY


def attn_last_error() -> str:
    return _lib().attn_last_error().decode()


def _check(status: int) -> None:
    if status != HYP_OK:
        raise HypError(status, attn_last_error())


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _int32(v: int, name: str) -> int:
    """v, where it fits the C int: ctypes would cut it."""
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError(f"{name}: {v} does not fit 32 bits")
    return v


def _ints(t: Optional[torch.Tensor], shape, name: str, index: int) -> Optional[int]:
    """The address of t, or None; index: the device's."""
    if t is None:
        return None
    if t.get_device() != index or t.dtype != torch.int32 or not t.is_contiguous() or tuple(t.shape) != shape:
        raise ValueError(f"{name}: need a contiguous int32 tensor {list(shape)} on the cache's device")
    return t.data_ptr()


class AttnCache:
    """Keys and values of n requests, and those that all of them share (hyp_attn_cache_t).

    k, v        [n, kv heads, most, d], or with page_table a pool [pages, kv heads, page keys, d]; f32 or bf16,
                any strides with contiguous features
    lens        [n] int32: own keys held
    page_table  [n, pages per request] int32
    most        bound on lens, by default the room there is
    prefix_k, prefix_v  [kv heads, prefix, d]
    key_pos, key_doc    [n, kv heads, most] int32, keys contiguous (heads may be expanded)
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor, page_table: Optional[torch.Tensor] = None,
                 most: Optional[int] = None, prefix_k: Optional[torch.Tensor] = None, prefix_v: Optional[torch.Tensor] = None,
                 key_pos: Optional[torch.Tensor] = None, key_doc: Optional[torch.Tensor] = None):
        _need(k.dim() == 4 and k.shape == v.shape, "k and v: need the same shape of four dimensions")
        _need(k.dtype in (torch.float32, torch.bfloat16), "k: need float32 or bfloat16")
        n, nkv, room, d = k.shape
        self.index = index = k.get_device()
        _need(k.is_cuda, "k: need a device tensor")
        for t, name in ((k, "k"), (v, "v"), (prefix_k, "prefix_k"), (prefix_v, "prefix_v")):
            _need(t is None or (t.get_device() == index and t.dtype == k.dtype and (t.stride(-1) == 1 or d == 1)), f"{name}: need a tensor of k's type on its device, features contiguous")
        c = _Cache()
        if page_table is not None:
            _need(page_table.dim() == 2, "page_table: need [requests, pages per request]")
            c.n_pages, c.page_keys, c.pages_per_request = _int32(n, "pages"), _int32(room, "page keys"), _int32(page_table.shape[1], "pages per request")
            n, room = page_table.shape[0], page_table.shape[1] * room
            c.page_table = _ints(page_table, tuple(page_table.shape), "page_table", index)
        self.most = _int32(room if most is None else int(most), "most")
        _need(self.most <= room, f"most: {self.most} keys, room for {room}")
        self.n_requests, self.n_kv_heads, self.head_dim, self.dtype, self.device = n, nkv, d, k.dtype, k.device
        c.k, c.v, c.most = k.data_ptr(), v.data_ptr(), self.most
        c.n_requests, c.n_kv_heads, c.head_dim = _int32(n, "requests"), _int32(nkv, "heads"), _int32(d, "features")
        c.k_page_stride, c.k_head_stride, c.k_key_stride = k.stride()[:3]
        c.v_page_stride, c.v_head_stride, c.v_key_stride = v.stride()[:3]
        c.dtype = HYP_BF16 if k.dtype == torch.bfloat16 else HYP_F32
        c.lens = _ints(lens, (n,), "lens", index)
        _need((prefix_k is None) == (prefix_v is None), "prefix_k and prefix_v go together")
        if prefix_k is not None:
            _need(prefix_k.dim() == 3 and prefix_k.shape == prefix_v.shape and (prefix_k.shape[0], prefix_k.shape[2]) == (nkv, d),
                  f"prefix_k and prefix_v: need [{nkv}, keys, {d}]")
            c.prefix_len = _int32(prefix_k.shape[1], "prefix")
            if c.prefix_len:
                c.prefix_k, c.prefix_v = prefix_k.data_ptr(), prefix_v.data_ptr()
            c.prefix_k_head_stride, c.prefix_k_key_stride = prefix_k.stride()[:2]
            c.prefix_v_head_stride, c.prefix_v_key_stride = prefix_v.stride()[:2]
        self.prefix_len = c.prefix_len
        for t, name in ((key_pos, "key_pos"), (key_doc, "key_doc")):
            if t is None:
                continue
            _need(t.get_device() == index and t.dtype == torch.int32 and t.dim() == 3 and tuple(t.shape[:2]) == (n, nkv) and t.shape[2] >= self.most
                  and (t.stride(2) == 1 or t.shape[2] == 1), f"{name}: need an int32 tensor [{n}, {nkv}, >= {self.most}] on k's device, keys contiguous")
            setattr(c, name, t.data_ptr())
            setattr(c, name + "_request_stride", t.stride(0))
            setattr(c, name + "_head_stride", t.stride(1))
        self._c, self._ref = c, C.byref(c)
        self._keep = (k, v, lens, page_table, prefix_k, prefix_v, key_pos, key_doc)


class AttnRule:
    """How scores are formed: scale * <q, k>, capped as cap * tanh(score / cap) (0: not), less slopes[head] * distance."""

    def __init__(self, scale: float, cap: float = 0.0, slopes: Optional[torch.Tensor] = None):
        _need(slopes is None or (slopes.is_cuda and slopes.dtype == torch.float32 and slopes.dim() == 1 and slopes.is_contiguous()),
              "slopes: need a contiguous float32 device tensor [query heads]")
        self.n_q_heads = None if slopes is None else slopes.shape[0]
        self.index = None if slopes is None else slopes.get_device()
        self._c = _Rule(float(scale), float(cap), None if slopes is None else slopes.data_ptr())
        self._ref, self._keep = C.byref(self._c), slopes


def _rows(cache: AttnCache, rule: AttnRule, q: torch.Tensor, q_start, see_all, q_pos, q_doc) -> _Rows:
    index = cache.index
    if q.dim() != 3 or q.dtype != cache.dtype or q.get_device() != index or q.shape[2] != cache.head_dim or (q.stride(2) != 1 and q.shape[2] != 1):
        raise ValueError(f"q: need a {cache.dtype} tensor [rows, query heads, {cache.head_dim}] on the cache's device, features contiguous")
    rows, heads = q.shape[0], q.shape[1]
    _need(rule.n_q_heads is None or (rule.n_q_heads == heads and rule.index == index), "slopes: need one for each query head, on the cache's device")
    return _Rows(q.data_ptr() or None, q.stride(0), q.stride(1), rows, _int32(heads, "query heads"),
                 None if q_start is None else _ints(q_start, (cache.n_requests + 1,), "q_start", index),
                 None if see_all is None else _ints(see_all, (cache.n_requests,), "see_all", index),
                 None if q_pos is None else _ints(q_pos, (rows,), "q_pos", index),
                 None if q_doc is None else _ints(q_doc, (rows,), "q_doc", index))


def _totals(cache: AttnCache, totals: torch.Tensor, totals_out: Optional[torch.Tensor], out_keys: int) -> _Totals:
    out = totals if totals_out is None else totals_out
    for t, keys, name in ((totals, cache.most, "totals"), (out, out_keys, "totals_out")):
        if (t.dim() != 3 or t.dtype != torch.float32 or t.get_device() != cache.index or t.shape[0] != cache.n_requests or t.shape[1] != cache.n_kv_heads
                or t.shape[2] < keys or (t.stride(2) != 1 and t.shape[2] != 1)):
            raise ValueError(f"{name}: need a float32 tensor [{cache.n_requests}, {cache.n_kv_heads}, >= {keys}] on the cache's device, keys contiguous")
    return _Totals(totals.data_ptr(), out.data_ptr(), totals.stride(0), totals.stride(1), out.stride(0), out.stride(1))


_HERE = contextlib.nullcontext()


def _on(stream):
    return _HERE if stream is None else torch.cuda.stream(stream)


def _handle(stream, index: int) -> int:
    if torch.cuda.current_device() != index:  # where the library launches; within _on(stream) the stream's
        raise ValueError("the cache's device is not the current one, or not the stream's")
    return _raw_stream(index) if stream is None else stream.cuda_stream


def _slow_raw_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


# the handle alone, without the Stream object around it, which takes a third of a small call's time
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _slow_raw_stream)


def _outputs(cache: AttnCache, q: torch.Tensor, out, lse):
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    elif out.shape != q.shape or out.dtype != q.dtype or out.get_device() != cache.index or (out.stride(2) != 1 and out.shape[2] != 1):
        raise ValueError("out: need a tensor of q's shape and type on its device, features contiguous")
    if lse is None:
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    elif lse.shape != q.shape[:2] or lse.dtype != torch.float32 or lse.get_device() != cache.index or not lse.is_contiguous():
        raise ValueError("lse: need a contiguous float32 tensor [rows, query heads] on the cache's device")
    return out, lse, _Out(out.data_ptr(), out.stride(0), out.stride(1), lse.data_ptr())


def _workspace(need: int, workspace: Optional[torch.Tensor], device) -> Tuple[Optional[torch.Tensor], Optional[int], int]:
    if workspace is None:
        if need == 0:
            return None, None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    elif workspace.device != device or not workspace.is_contiguous():
        raise ValueError("workspace: need a contiguous tensor on the cache's device")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def attn_workspace_bytes(cache: AttnCache, rule: AttnRule, q: torch.Tensor, q_start: Optional[torch.Tensor] = None, totals: bool = False) -> int:
    """Bytes of workspace of attn_prompt (q_start given) or attn_token for rows like q."""
    t = _Totals()
    return int(_lib().attn_workspace_bytes(cache._ref, C.byref(_rows(cache, rule, q, q_start, None, None, None)), C.byref(t) if totals else None))


def attn_prompt(cache: AttnCache, rule: AttnRule, q: torch.Tensor, q_start: torch.Tensor, see_all: Optional[torch.Tensor] = None,
                q_pos: Optional[torch.Tensor] = None, q_doc: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(out, lse) of the newest rows of every request: request b has rows q_start[b] .. q_start[b + 1] - 1 of q."""
    lib = _lib()
    with _on(stream):
        rows = _rows(cache, rule, q, q_start, see_all, q_pos, q_doc)
        out, lse, o = _outputs(cache, q, out, lse)
        need = lib.attn_workspace_bytes(cache._ref, C.byref(rows), None) if workspace is None else 0
        workspace, ptr, size = _workspace(need, workspace, cache.device)
        _check(lib.attn_prompt(cache._ref, rule._ref, C.byref(rows), C.byref(o), ptr, size, _handle(stream, cache.index)))
    return out, lse


def attn_token(cache: AttnCache, rule: AttnRule, q: torch.Tensor, q_pos: Optional[torch.Tensor] = None, q_doc: Optional[torch.Tensor] = None,
               totals: Optional[torch.Tensor] = None, totals_out: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(out, lse) of one row a request, its newest key; the weight that own keys got is added to totals (in place, or into totals_out)."""
    lib = _lib()
    with _on(stream):
        rows = _rows(cache, rule, q, None, None, q_pos, q_doc)
        out, lse, o = _outputs(cache, q, out, lse)
        t = None if totals is None else C.byref(_totals(cache, totals, totals_out, cache.most))
        need = lib.attn_workspace_bytes(cache._ref, C.byref(rows), t) if workspace is None else 0
        workspace, ptr, size = _workspace(need, workspace, cache.device)
        _check(lib.attn_token(cache._ref, rule._ref, C.byref(rows), C.byref(o), t, ptr, size, _handle(stream, cache.index)))
    return out, lse


def attn_received(cache: AttnCache, rule: AttnRule, q: torch.Tensor, q_start: torch.Tensor, lse: torch.Tensor, totals: torch.Tensor, last: int = 0,
                  see_all: Optional[torch.Tensor] = None, q_pos: Optional[torch.Tensor] = None, q_doc: Optional[torch.Tensor] = None,
                  totals_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Adds the weight that own keys got from each request's last rows (0: all) to totals (in place, or into totals_out); lse: attn_prompt's."""
    with _on(stream):
        rows = _rows(cache, rule, q, q_start, see_all, q_pos, q_doc)
        if lse.shape != q.shape[:2] or lse.dtype != torch.float32 or lse.get_device() != cache.index or not lse.is_contiguous():
            raise ValueError("lse: need a contiguous float32 tensor [rows, query heads] on the cache's device")
        t = _totals(cache, totals, totals_out, cache.most)
        _check(_lib().attn_received(cache._ref, rule._ref, C.byref(rows), lse.data_ptr(), _int32(last, "last"), C.byref(t), _handle(stream, cache.index)))
    return totals if totals_out is None else totals_out


def attn_evict_workspace_bytes(cache: AttnCache, keep: int) -> int:
    """Bytes of workspace of attn_evict."""
    return int(_lib().attn_evict_workspace_bytes(cache._ref, _int32(keep, "keep")))


def attn_evict(cache: AttnCache, totals: torch.Tensor, keep: int, sink: int = 0, recent: int = 0, now: Optional[torch.Tensor] = None,
               into: Optional[AttnCache] = None, totals_out: Optional[torch.Tensor] = None, kept: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Keeps at most `keep` keys of every request and KV head, in place or into another cache; returns the slots they came from
    [n, kv heads, keep] (-1: none)."""
    lib = _lib()
    for value, name in ((keep, "keep"), (sink, "sink"), (recent, "recent")):
        _int32(value, name)
    _need((into is None) == (totals_out is None), "totals_out goes with into")
    _need(into is None or into.index == cache.index, "into: need a cache on the same device")
    with _on(stream):
        if kept is None:
            kept = torch.empty((cache.n_requests, cache.n_kv_heads, max(keep, 0)), dtype=torch.int32, device=cache.device)
        t = _totals(cache, totals, totals_out, 0 if into is None else keep)
        need = lib.attn_evict_workspace_bytes(cache._ref, keep) if workspace is None else 0
        workspace, ptr, size = _workspace(need, workspace, cache.device)
        _check(lib.attn_evict(cache._ref, None if into is None else into._ref, C.byref(t), keep, sink, recent,
                              None if now is None else _ints(now, (cache.n_requests,), "now", cache.index),
                              _ints(kept, (cache.n_requests, cache.n_kv_heads, max(keep, 0)), "kept", cache.index), ptr, size, _handle(stream, cache.index)))
    return kept
