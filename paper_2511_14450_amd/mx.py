"""ctypes binding of include/hyp_mx.h: caches of keys and values in 8 or 4 bits, and single tokens that read them whole or in selected blocks.

Same names as the C ABI, argument marshalling only; PyTorch owns the memory and the streams.  Work is
enqueued on `stream` (default: torch's current one), and so is the allocation of what a call returns.
An MxCache describes tensors that the caller goes on owning: rows are written by mx_write, after the
caller has counted them in lens.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from .attn import AttnRule, _handle, _int32, _ints, _need, _on, _Out, _Rule, _workspace
from .binding import HYP_BF16, HYP_F32, HYP_OK, HypError, load_library

EXPORTS_MX = ("mx_write", "mx_read", "mx_select_workspace_bytes", "mx_select", "mx_token_workspace_bytes", "mx_token", "mx_last_error")
HYP_E4M3, HYP_E2M1 = 0, 1
MX_FORMATS = {"e4m3": HYP_E4M3, "e2m1": HYP_E2M1}
_GROUP_BYTES = (32, 16)
_DTYPES = {torch.float32: HYP_F32, torch.bfloat16: HYP_BF16}


class _MxCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("k_page_stride", C.c_int64), ("k_head_stride", C.c_int64), ("k_key_stride", C.c_int64),
                ("v_page_stride", C.c_int64), ("v_head_stride", C.c_int64), ("v_key_stride", C.c_int64),
                ("k_scale_page_stride", C.c_int64), ("k_scale_head_stride", C.c_int64), ("k_scale_group_stride", C.c_int64),
                ("v_scale_page_stride", C.c_int64), ("v_scale_head_stride", C.c_int64), ("v_scale_group_stride", C.c_int64),
                ("page_table", C.c_void_p), ("pages_per_request", C.c_int32), ("page_keys", C.c_int32), ("n_pages", C.c_int32),
                ("lens", C.c_void_p), ("most", C.c_int32),
                ("n_requests", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("k_format", C.c_int32), ("v_format", C.c_int32),
                ("lo", C.c_void_p), ("hi", C.c_void_p),
                ("bound_page_stride", C.c_int64), ("bound_head_stride", C.c_int64), ("bound_block_stride", C.c_int64), ("block_keys", C.c_int32)]


class _MxRows(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p),
                ("k_row_stride", C.c_int64), ("k_head_stride", C.c_int64), ("v_row_stride", C.c_int64), ("v_head_stride", C.c_int64),
                ("k_out", C.c_void_p), ("v_out", C.c_void_p),
                ("k_out_row_stride", C.c_int64), ("k_out_head_stride", C.c_int64), ("v_out_row_stride", C.c_int64), ("v_out_head_stride", C.c_int64),
                ("n_rows", C.c_int64), ("q_start", C.c_void_p), ("dtype", C.c_int32)]


class _MxOut(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p),
                ("k_request_stride", C.c_int64), ("k_head_stride", C.c_int64), ("k_key_stride", C.c_int64),
                ("v_request_stride", C.c_int64), ("v_head_stride", C.c_int64), ("v_key_stride", C.c_int64), ("keys", C.c_int32), ("dtype", C.c_int32)]


class _MxQ(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_row_stride", C.c_int64), ("q_head_stride", C.c_int64), ("n_q_heads", C.c_int32), ("dtype", C.c_int32)]


_READY = None


def _lib() -> C.CDLL:
    global _READY
    if _READY is None:
        lib = load_library()
        cache, rows, to, q, rule, out = (C.POINTER(t) for t in (_MxCache, _MxRows, _MxOut, _MxQ, _Rule, _Out))
        lib.mx_write.restype = C.c_int
        lib.mx_write.argtypes = [cache, rows, C.c_void_p]
        lib.mx_read.restype = C.c_int
        lib.mx_read.argtypes = [cache, C.c_void_p, to, C.c_void_p]
        lib.mx_select_workspace_bytes.restype = C.c_size_t
        lib.mx_select_workspace_bytes.argtypes = [cache, q, C.c_int32]
        lib.mx_select.restype = C.c_int
        lib.mx_select.argtypes = [cache, q, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.mx_token_workspace_bytes.restype = C.c_size_t
        lib.mx_token_workspace_bytes.argtypes = [cache, q, C.c_int32]
        lib.mx_token.restype = C.c_int
        lib.mx_token.argtypes = [cache, rule, q, C.c_void_p, C.c_int32, out, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.mx_last_error.restype = C.c_char_p
        lib.mx_last_error.argtypes = []
        _READY = lib
    return _READY


def mx_last_error() -> str:
    return _lib().mx_last_error().decode()


def _check(status: int) -> None:
    if status != HYP_OK:
        raise HypError(status, mx_last_error())


class MxCache:
    """Keys and values of n requests in 8 or 4 bits a feature (hyp_mx_cache_t).

    k, v              codes, uint8 [n, kv heads, room, width], or with page_table a pool [pages, kv heads, page keys, width], codes of a key contiguous;
                      width is 32 ("e4m3") or 16 ("e2m1") for each group of 32 features, which gives the format; room is a multiple of 16
    k_scale, v_scale  uint8 [n or pages, kv heads, groups, room or page keys], keys contiguous
    lens              [n] int32: keys held
    head_dim          features, of which ceil(head_dim / 32) groups are kept
    page_table        [n, pages per request] int32
    most              bound on lens, by default the room there is
    lo, hi            bfloat16 [n or pages, kv heads, blocks of the room or page, head_dim], both with the same strides, features contiguous: bounds that
                      mx_write keeps and mx_select reads
    block_keys        keys of a block (0: none), by default what lo says
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, lens: torch.Tensor, head_dim: int,
                 page_table: Optional[torch.Tensor] = None, most: Optional[int] = None, lo: Optional[torch.Tensor] = None,
                 hi: Optional[torch.Tensor] = None, block_keys: Optional[int] = None):
        _need(k.is_cuda, "k: need a device tensor")
        self.index = index = k.get_device()
        self.head_dim, self.device = int(head_dim), k.device
        _need(1 <= self.head_dim <= 256, "head_dim: need 1..256")
        groups = -(-self.head_dim // 32)
        _need(k.dim() == 4 and v.dim() == 4 and k.shape[:3] == v.shape[:3], "k and v: need four dimensions, the first three the same")
        n, nkv, room = k.shape[:3]
        c = _MxCache()
        for t, name in ((k, "k"), (v, "v")):
            _need(t.get_device() == index and t.dtype == torch.uint8 and t.stride(3) == 1, f"{name}: need a uint8 tensor on k's device, codes of a key contiguous")
            _need(t.shape[3] in (32 * groups, 16 * groups), f"{name}: need {32 * groups} (e4m3) or {16 * groups} (e2m1) bytes a key")
            setattr(c, name + "_format", HYP_E4M3 if t.shape[3] == 32 * groups else HYP_E2M1)
            setattr(c, name, t.data_ptr())
            for i, what in enumerate(("page", "head", "key")):
                setattr(c, f"{name}_{what}_stride", t.stride(i))
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _need(t.get_device() == index and t.dtype == torch.uint8 and tuple(t.shape) == (n, nkv, groups, room) and (t.stride(3) == 1 or room == 1),
                  f"{name}: need a uint8 tensor {[n, nkv, groups, room]} on k's device, keys contiguous")
            setattr(c, name, t.data_ptr())
            for i, what in enumerate(("page", "head", "group")):
                setattr(c, f"{name}_{what}_stride", t.stride(i))
        c.page_keys = _int32(room, "keys")
        pages = n
        if page_table is not None:
            _need(page_table.dim() == 2, "page_table: need [requests, pages per request]")
            c.n_pages, c.pages_per_request = _int32(n, "pages"), _int32(page_table.shape[1], "pages per request")
            c.page_table = _ints(page_table, tuple(page_table.shape), "page_table", index)
            n, room = page_table.shape[0], page_table.shape[1] * room
        self.most = _int32(room if most is None else int(most), "most")
        _need(self.most <= room, f"most: {self.most} keys, room for {room}")
        self.n_requests, self.n_kv_heads = n, nkv
        c.most, c.n_requests, c.n_kv_heads, c.head_dim = self.most, _int32(n, "requests"), _int32(nkv, "heads"), self.head_dim
        c.lens = _ints(lens, (n,), "lens", index)
        _need((lo is None) == (hi is None), "lo and hi go together")
        if lo is not None:
            for t, name in ((lo, "lo"), (hi, "hi")):
                _need(t.get_device() == index and t.dtype == torch.bfloat16 and t.dim() == 4 and (t.shape[0], t.shape[1], t.shape[3]) == (pages, nkv, self.head_dim)
                      and (t.stride(3) == 1 or self.head_dim == 1) and t.shape[2] >= 1 and c.page_keys % t.shape[2] == 0,
                      f"{name}: need a bfloat16 tensor [{pages}, {nkv}, blocks, {self.head_dim}] on k's device, features contiguous")
            _need(lo.shape == hi.shape and lo.stride() == hi.stride(), "lo and hi: need the same shape and strides")
            blocks = c.page_keys // lo.shape[2]
            _need(block_keys is None or block_keys == blocks, f"block_keys: lo and hi are of blocks of {blocks} keys")
            block_keys = blocks
            c.lo, c.hi = lo.data_ptr(), hi.data_ptr()
            c.bound_page_stride, c.bound_head_stride, c.bound_block_stride = lo.stride()[:3]
        self.block_keys = c.block_keys = _int32(block_keys or 0, "block_keys")
        self._c, self._ref = c, C.byref(c)
        self._keep = (k, v, k_scale, v_scale, lens, page_table, lo, hi)

    @classmethod
    def allocate(cls, n_requests: int, n_kv_heads: int, most: int, head_dim: int, k_format: str = "e4m3", v_format: str = "e4m3", block_keys: int = 0,
                 page_keys: int = 0, n_pages: Optional[int] = None, lens: Optional[torch.Tensor] = None, page_table: Optional[torch.Tensor] = None,
                 device="cuda") -> "MxCache":
        """An empty cache with memory of its own: slabs, or pages of page_keys keys (n_pages of them, by default enough for all; request b has pages
        b * ceil(most / page_keys) on until the caller writes another table, and with fewer pages than that takes the caller has to give one).  block_keys > 0: with bounds of such blocks.  lens, page_table: where
        several caches, of a model's blocks, share them.  Its tensors are the attributes k, v, k_scale, v_scale, lens, page_table, lo and hi."""
        for name in (k_format, v_format):
            _need(name in MX_FORMATS, f"format: need one of {', '.join(MX_FORMATS)}")
        groups, unit, table = -(-head_dim // 32), max(16, block_keys), page_table
        _need(page_table is None or page_keys, "page_table goes with page_keys")
        if page_keys:
            per = -(-most // page_keys)
            slabs, room = n_requests * per if n_pages is None else n_pages, page_keys
            if table is None:
                _need(slabs >= n_requests * per, f"n_pages: {slabs} pages are not enough for all requests, which have {n_requests * per}: give a page_table")
                table = torch.arange(n_requests * per, dtype=torch.int32, device=device).reshape(n_requests, per)
        else:
            slabs, room = n_requests, -(-most // unit) * unit
        _need(block_keys == 0 or (16 <= block_keys <= 4096 and block_keys & (block_keys - 1) == 0 and room % block_keys == 0),
              f"block_keys: need a power of two from 16 to 4096{f' that divides page_keys, {page_keys}' if page_keys else ''}")
        new = lambda *shape, dtype=torch.uint8: torch.zeros(shape, dtype=dtype, device=device)  # noqa: E731
        k, v = (new(slabs, n_kv_heads, room, _GROUP_BYTES[MX_FORMATS[f]] * groups) for f in (k_format, v_format))
        k_scale, v_scale = (new(slabs, n_kv_heads, groups, room) for _ in range(2))
        lo, hi = (new(slabs, n_kv_heads, room // block_keys, head_dim, dtype=torch.bfloat16) if block_keys else None for _ in range(2))
        return cls(k, v, k_scale, v_scale, new(n_requests, dtype=torch.int32) if lens is None else lens, head_dim, page_table=table, most=most, lo=lo, hi=hi)

    k, v, k_scale, v_scale, lens, page_table, lo, hi = (property(lambda self, i=i: self._keep[i]) for i in range(8))


def _features(t: torch.Tensor, d: int) -> bool:
    return t.stride(-1) == 1 or d == 1


def mx_write(cache: MxCache, k: torch.Tensor, v: torch.Tensor, q_start: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
             v_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Quantises rows [rows, kv heads, d] (f32 or bf16), the newest keys of every request, into the cache: request b has rows q_start[b] ..
    q_start[b + 1] - 1 (no q_start: row b); the numbers that are stored also go to k_out and v_out, which may be k and v."""
    index, nkv, d = cache.index, cache.n_kv_heads, cache.head_dim
    shape, dtype = k.shape, k.dtype
    _need((k_out is None) == (v_out is None), "k_out and v_out go together")
    for t, name in ((k, "k"), (v, "v")) if k_out is None else ((k, "k"), (v, "v"), (k_out, "k_out"), (v_out, "v_out")):
        if len(shape) != 3 or t.shape != shape or t.dtype != dtype or t.get_device() != index or (t.stride(2) != 1 and d != 1):
            raise ValueError(f"{name}: need a tensor of k's shape and type on the cache's device, features contiguous")
    if dtype not in _DTYPES or shape[1] != nkv or shape[2] != d:
        raise ValueError(f"k: need a float32 or bfloat16 tensor [rows, {nkv}, {d}]")
    ks, vs = k.stride(), v.stride()
    start = None if q_start is None else _ints(q_start, (cache.n_requests + 1,), "q_start", index)
    if k_out is None:
        rows = _MxRows(k.data_ptr(), v.data_ptr(), ks[0], ks[1], vs[0], vs[1], None, None, 0, 0, 0, 0, shape[0], start, _DTYPES[dtype])
    else:
        ko, vo = k_out.stride(), v_out.stride()
        rows = _MxRows(k.data_ptr(), v.data_ptr(), ks[0], ks[1], vs[0], vs[1], k_out.data_ptr(), v_out.data_ptr(), ko[0], ko[1], vo[0], vo[1], shape[0], start, _DTYPES[dtype])
    with _on(stream):
        _check(_lib().mx_write(cache._ref, C.byref(rows), _handle(stream, index)))


def mx_read(cache: MxCache, k: torch.Tensor, v: torch.Tensor, first: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Numbers of the keys first[b] (by default 0) .. lens[b] - 1 of every request b to k and v [n, kv heads, keys, d] (f32 or bf16, any strides with
    contiguous features), as many as there is room for; what lies behind them stays as it is."""
    index, d = cache.index, cache.head_dim
    for t, name in ((k, "k"), (v, "v")):
        if (t.dim() != 4 or t.shape != k.shape or t.dtype != k.dtype or t.get_device() != index or tuple(t.shape[:2]) != (cache.n_requests, cache.n_kv_heads)
                or t.shape[3] != d or t.dtype not in _DTYPES or not _features(t, d)):
            raise ValueError(f"{name}: need a float32 or bfloat16 tensor [{cache.n_requests}, {cache.n_kv_heads}, keys, {d}] on the cache's device, features contiguous, k and v alike")
    to = _MxOut(k.data_ptr(), v.data_ptr(), *k.stride()[:3], *v.stride()[:3], _int32(k.shape[2], "keys"), _DTYPES[k.dtype])
    with _on(stream):
        _check(_lib().mx_read(cache._ref, None if first is None else _ints(first, (cache.n_requests,), "first", index), C.byref(to), _handle(stream, index)))


def _q(cache: MxCache, q: torch.Tensor) -> _MxQ:
    shape, stride, d = q.shape, q.stride(), cache.head_dim
    if (len(shape) != 3 or q.dtype not in _DTYPES or q.get_device() != cache.index or shape[0] != cache.n_requests or shape[2] != d
            or (stride[2] != 1 and d != 1)):
        raise ValueError(f"q: need a float32 or bfloat16 tensor [{cache.n_requests}, query heads, {d}] on the cache's device, features contiguous")
    return _MxQ(q.data_ptr(), stride[0], stride[1], _int32(shape[1], "query heads"), _DTYPES[q.dtype])


def mx_select_workspace_bytes(cache: MxCache, q: torch.Tensor, keep: int) -> int:
    """Bytes of workspace of mx_select."""
    return int(_lib().mx_select_workspace_bytes(cache._ref, C.byref(_q(cache, q)), _int32(keep, "keep")))


def mx_select(cache: MxCache, q: torch.Tensor, keep: int, sink: int = 0, recent: int = 0, blocks: Optional[torch.Tensor] = None,
              workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The blocks [n, kv heads, keep] (int32, ascending, -1 behind the last) whose keys can have the largest scores with the rows q [n, query heads, d]."""
    lib = _lib()
    for value, name in ((keep, "keep"), (sink, "sink"), (recent, "recent")):
        _int32(value, name)
    with _on(stream):
        row = C.byref(_q(cache, q))
        shape = (cache.n_requests, cache.n_kv_heads, max(keep, 0))
        if blocks is None:
            blocks = torch.empty(shape, dtype=torch.int32, device=cache.device)
        need = lib.mx_select_workspace_bytes(cache._ref, row, keep) if workspace is None else 0
        workspace, ptr, size = _workspace(need, workspace, cache.device)
        _check(lib.mx_select(cache._ref, row, keep, sink, recent, _ints(blocks, shape, "blocks", cache.index), ptr, size, _handle(stream, cache.index)))
    return blocks


def mx_token_workspace_bytes(cache: MxCache, q: torch.Tensor, listed: int = 0) -> int:
    """Bytes of workspace of mx_token over so many listed blocks (0: all keys)."""
    return int(_lib().mx_token_workspace_bytes(cache._ref, C.byref(_q(cache, q)), _int32(listed, "listed")))


def mx_token(cache: MxCache, rule: AttnRule, q: torch.Tensor, blocks: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
             lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(out, lse) of one row a request, q [n, query heads, d], its newest key: over all keys, or over those of blocks [n, kv heads, listed] (int32)."""
    lib, index = _lib(), cache.index
    with _on(stream):
        row, shape = C.byref(_q(cache, q)), q.shape
        if rule.n_q_heads is not None and (rule.n_q_heads != shape[1] or rule.index != index):
            raise ValueError("slopes: need one for each query head, on the cache's device")
        listed, ptr = 0, None
        if blocks is not None:
            _need(blocks.dim() == 3 and blocks.shape[2] >= 1, "blocks: need [requests, kv heads, blocks]")
            listed = _int32(blocks.shape[2], "blocks")
            ptr = _ints(blocks, (cache.n_requests, cache.n_kv_heads, listed), "blocks", index)
        if out is None:
            out = torch.empty_like(q)  # of a dense q with its order of strides, else contiguous
        elif out.shape != shape or out.dtype != q.dtype or out.get_device() != index or not _features(out, cache.head_dim):
            raise ValueError("out: need a tensor of q's shape and type on its device, features contiguous")
        if lse is None:
            lse = q.new_empty(shape[:2], dtype=torch.float32)
        elif lse.shape != shape[:2] or lse.dtype != torch.float32 or lse.get_device() != index or not lse.is_contiguous():
            raise ValueError("lse: need a contiguous float32 tensor [requests, query heads] on the cache's device")
        work, size = None, 0
        if workspace is not None or (size := lib.mx_token_workspace_bytes(cache._ref, row, listed)):
            workspace, work, size = _workspace(size, workspace, cache.device)
        stride = out.stride()
        status = lib.mx_token(cache._ref, rule._ref, row, ptr, listed, C.byref(_Out(out.data_ptr(), stride[0], stride[1], lse.data_ptr())), work, size, _handle(stream, index))
        if status:
            _check(status)
    return out, lse
