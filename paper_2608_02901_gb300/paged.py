"""Binding of the paged 4-bit cache (the akv_paged_* and akv_pages_* entry points of ``include/akv.h``).

Argument marshalling only, like the rest of the package, which re-exports every name here.  A program makes
PagedParams and Pages once and calls with them; Pages keeps the C structures, so that a call of a decode loop
converts only what changes.

A serving loop: akv_pages_reserve, akv_paged_append, akv_pages_share (where rows are forks of others), then akv_paged_attn or
akv_paged_attn_shared, or akv_paged_select and akv_paged_attn over what it keeps.  For rows of bounded length: akv_paged_weights after the attention, and now
and then akv_paged_evict and akv_pages_trim.
"""
from __future__ import annotations

import ctypes
from contextlib import nullcontext
from dataclasses import dataclass, replace

AKV_FLAG_BOUNDS = 8
AKV_DTYPE_BF16, AKV_DTYPE_FP16 = 0, 1
AKV_SHARE_ALWAYS = 1
AKV_PAGED_MAX_QUERY = 64

EXPORTED = (
    "akv_paged_page_bytes", "akv_paged_append", "akv_paged_read", "akv_paged_attn_workspace_size", "akv_paged_attn",
    "akv_paged_select_workspace_size", "akv_paged_select", "akv_pages_copy", "akv_pages_fork",
    "akv_pages_workspace_size", "akv_pages_reserve", "akv_pages_free", "akv_pages_compact", "akv_pages_share",
    "akv_paged_attn_shared_workspace_size", "akv_paged_attn_shared", "akv_paged_weights_workspace_size", "akv_paged_weights",
    "akv_paged_evict", "akv_pages_trim",
)

_vp, _i32, _i64, _sz, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float


class _PagedParams(ctypes.Structure):
    _fields_ = [("n_kv_heads", _i32), ("n_q_heads", _i32), ("head_dim", _i32), ("page_tokens", _i32), ("group", _i32),
                ("dtype", _i32), ("flags", ctypes.c_uint32), ("reserved", _i32), ("rot_seed", ctypes.c_uint64)]


class _Pages(ctypes.Structure):
    _fields_ = [("pool", _vp), ("pool_bytes", _sz), ("layer_stride", _sz), ("n_layers", _i32), ("n_pages", _i32),
                ("table", _vp), ("table_stride", _i64), ("rows", _i32), ("max_pages", _i32), ("lens", _vp),
                ("refs", _vp)]


class _Rows(ctypes.Structure):
    _fields_ = [("ptr", _vp), ("stride_b", _i64), ("stride_t", _i64), ("stride_h", _i64)]


class _Selection(ctypes.Structure):
    _fields_ = [("pages", _vp), ("count", _vp), ("top", _i32)]


class _Share(ctypes.Structure):
    _fields_ = [("leader", _vp), ("pages", _vp), ("size", _vp), ("order", _vp), ("flags", ctypes.c_uint32)]


class _Scores(ctypes.Structure):
    _fields_ = [("ptr", _vp), ("stride_b", _i64), ("stride_h", _i64), ("cap", _i32)]


class _Kept(ctypes.Structure):
    _fields_ = [("tokens", _vp), ("count", _vp), ("top", _i32)]


def declare(L):
    """Argument types of the entry points in a loaded libakv.so."""
    P, G, R, S, H, N, K = (ctypes.POINTER(t) for t in (_PagedParams, _Pages, _Rows, _Selection, _Share, _Scores, _Kept))
    out = ctypes.POINTER(_sz)
    for name, args in (
            ("akv_paged_page_bytes", [P, out]),
            ("akv_paged_append", [P, G, _i32, R, R, _i32, _vp, _vp]),
            ("akv_paged_read", [P, G, _i32, _vp, R, R, _i32, _vp]),
            ("akv_paged_attn_workspace_size", [P, G, _i32, _i32, out]),
            ("akv_paged_attn", [P, G, _i32, R, R, _vp, _i32, _f32, S, _vp, _sz, _vp]),
            ("akv_paged_select_workspace_size", [P, G, _i32, out]),
            ("akv_paged_select", [P, G, _i32, R, _i32, _i32, _i32, S, _vp, _sz, _vp]),
            ("akv_pages_copy", [P, G, _vp, _vp, _i32, _vp]),
            ("akv_pages_fork", [P, G, _vp, _vp, _i32, _vp]),
            ("akv_pages_workspace_size", [P, G, out]),
            ("akv_pages_reserve", [P, G, _vp, _vp, _vp, _sz, _vp]),
            ("akv_pages_free", [P, G, _vp, _i32, _vp]),
            ("akv_pages_compact", [P, G, _vp, _vp, _sz, _vp]),
            ("akv_pages_share", [P, G, H, _vp, _sz, _vp]),
            ("akv_paged_attn_shared_workspace_size", [P, G, _i32, out]),
            ("akv_paged_attn_shared", [P, G, _i32, R, R, _vp, _i32, _f32, H, _vp, _sz, _vp]),
            ("akv_paged_weights_workspace_size", [P, G, _i32, out]),
            ("akv_paged_weights", [P, G, _i32, R, _vp, _i32, _f32, _f32, N, N, _vp, _sz, _vp]),
            ("akv_paged_evict", [P, G, _i32, _vp, _vp, _i32, N, _vp, _i32, _i32, K, _vp]),
            ("akv_pages_trim", [P, G, _vp, _i32, _vp])):
        f = getattr(L, name)
        f.restype, f.argtypes = ctypes.c_int, args


@dataclass(frozen=True)
class PagedParams:
    """A paged cache's heads and codec (see akv_paged_params in include/akv.h)."""
    n_kv_heads: int
    n_q_heads: int
    page_tokens: int = 64
    group: int = 64
    half: bool = False  # fp16 rows instead of bf16
    rotate: bool = True
    bounds: bool = False  # pages carry their keys' bounds, for akv_paged_select
    rot_seed: int = 0x5EED
    head_dim: int = 128

    @property
    def G(self) -> int:
        return self.n_q_heads // self.n_kv_heads

    def c(self) -> _PagedParams:
        from . import AKV_FLAG_ROTATE
        return _PagedParams(self.n_kv_heads, self.n_q_heads, self.head_dim, self.page_tokens, self.group,
                            AKV_DTYPE_FP16 if self.half else AKV_DTYPE_BF16,
                            (AKV_FLAG_ROTATE if self.rotate else 0) | (AKV_FLAG_BOUNDS if self.bounds else 0), 0,
                            self.rot_seed & (2**64 - 1))


def akv_paged_page_bytes(p: PagedParams) -> int:
    n = _sz()
    _check(_lib().akv_paged_page_bytes(ctypes.byref(p.c()), ctypes.byref(n)), "akv_paged_page_bytes")
    return n.value


_loaded = None
_torch = _bf16 = _fp16 = _int32 = _raw_stream = _device = None


def _lib():
    """The library; torch is loaded with it."""
    global _loaded, _torch, _bf16, _fp16, _int32, _raw_stream, _device
    if _loaded is None:
        import torch

        from . import lib
        _torch, _bf16, _fp16, _int32 = torch, torch.bfloat16, torch.float16, torch.int32
        _raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        _loaded = lib()
    return _loaded


def _check(status, where):
    if status:
        from . import _check as check
        check(status, where)


def _stream(stream, pages):
    """Address of a stream: the current one of the pool's device for None."""
    if stream is None:
        return _raw_stream(pages.index)
    if getattr(stream, "device_index", pages.index) != pages.index:
        raise ValueError("stream must be one of the pool's device")
    return getattr(stream, "cuda_stream", stream)


def _there(pages, call, *args):
    """The call with the pool's device as the current one: entries launch on that."""
    with _torch.cuda.device(pages.index):
        return call(*args)


def _ints(t, what, n, index):
    """Address of a contiguous CUDA int32 tensor of n elements (None: any number) on device `index`, or None for None."""
    if t is None:
        return None
    if t.dtype is not _int32 or t.get_device() != index or not t.is_contiguous() or (n is not None and t.numel() != n):
        raise ValueError(f"{what} must be a contiguous CUDA int32 tensor on the pool's device"
                         + ("" if n is None else f" and hold {n} numbers"))
    return t.data_ptr()


class Pages:
    """The pages of a cache: CUDA tensors that the caller owns and keeps alive.

    pool   [n_layers][n_pages][...] of any type, each page's bytes (akv_paged_page_bytes) contiguous and next to
           the page before; layers may lie further apart
    table  int32 [rows][max_pages], rows may lie further apart: the page of each page_tokens tokens, -1 = none
    lens   int32 [rows]: tokens held
    refs   int32 [n_pages]: holders of each page, 0 = free; needed by akv_pages_fork, _reserve, _free and _compact, and
           where given akv_paged_append writes to no page with more than one
    """

    def __init__(self, p: PagedParams, pool, table, lens, refs=None):
        page = akv_paged_page_bytes(p)  # (loads the library)
        if not pool.is_cuda or pool.dim() < 2:
            raise ValueError("pool must be a CUDA tensor [n_layers][n_pages][...]")
        n_layers, n_pages = int(pool.shape[0]), int(pool.shape[1])
        if pool[0].numel() * pool.element_size() != n_pages * page or not pool[0].is_contiguous():
            raise ValueError(f"pool must hold pages of {page} contiguous bytes")
        if not table.is_cuda or table.dtype is not _int32 or table.dim() != 2 or table.stride(1) != 1:
            raise ValueError("table must be a CUDA int32 tensor [rows][max_pages] with adjacent columns")
        if table.device != pool.device:
            raise ValueError("table must be on the pool's device")
        rows, most = table.shape
        self.p, self.pool, self.table, self.lens, self.refs = p, pool, table, lens, refs
        self.rows, self.max_pages, self.n_layers, self.n_pages, self.device = rows, most, n_layers, n_pages, pool.device
        self.index = pool.device.index
        stride = pool.stride(0) * pool.element_size() if n_layers > 1 else n_pages * page
        self._params = p.c()
        self._c = _Pages(pool.data_ptr(), (n_layers - 1) * stride + n_pages * page, stride, n_layers, n_pages,
                         table.data_ptr(), table.stride(0) if rows > 1 else max(table.stride(0), most), rows, most,
                         _ints(lens, "lens", rows, self.index), _ints(refs, "refs", n_pages, self.index))
        self.pref, self.ref = ctypes.byref(self._params), ctypes.byref(self._c)


class PageSelection:
    """Pages kept for each query token and KV head: CUDA int32 pages [rows][T][n_kv_heads][top], count
    [rows][T][n_kv_heads], both contiguous."""

    def __init__(self, pages, count):
        if pages.dim() != 4 or tuple(count.shape) != tuple(pages.shape[:3]):
            raise ValueError("selection: pages [rows][T][n_kv_heads][top] and count [rows][T][n_kv_heads]")
        self.pages, self.count, self.top = pages, count, int(pages.shape[3])
        _lib()
        self._c = _Selection(_ints(pages, "selection pages", None, pages.get_device()),
                             _ints(count, "selection count", None, pages.get_device()), self.top)
        self.ref = ctypes.byref(self._c)


class PageShare:
    """Rows that begin with the same pages, as akv_pages_share finds them: a contiguous CUDA int32 tensor [4][rows] of
    leader, pages, size and order (akv_share in include/akv.h).  always: akv_paged_attn_shared reads every group's pages once, also where
    row by row is faster."""

    def __init__(self, arrays, always: bool = False):
        if arrays.dim() != 2 or arrays.shape[0] != 4:
            raise ValueError("share must be [4][rows]")
        _lib()
        self.arrays, self.rows, self.index = arrays, int(arrays.shape[1]), arrays.get_device()
        at = _ints(arrays, "share", None, self.index)
        if self.index < 0:
            raise ValueError("share must be on the pool's device")
        self._c = _Share(*(at + 4 * self.rows * i for i in range(4)), AKV_SHARE_ALWAYS if always else 0)
        self.ref = ctypes.byref(self._c)


class KeptTokens:
    """Tokens that rows keep: CUDA int32 tokens [n][n_kv_heads][top], count [n], both contiguous."""

    def __init__(self, tokens, count):
        if tokens.dim() != 3 or tuple(count.shape) != (tokens.shape[0],):
            raise ValueError("kept: tokens [n][n_kv_heads][top] and count [n]")
        self.tokens, self.count, self.top = tokens, count, int(tokens.shape[2])
        _lib()
        self._c = _Kept(_ints(tokens, "kept tokens", None, tokens.get_device()),
                        _ints(count, "kept count", None, tokens.get_device()), self.top)
        self.ref = ctypes.byref(self._c)


def _params(p: PagedParams, pages: Pages):
    """The C parameters of p, which describes the pool's pages (its query heads may differ)."""
    if p is pages.p:
        return pages.pref
    if replace(p, n_q_heads=pages.p.n_q_heads) != pages.p:
        raise ValueError("the parameters are not those of the pool's pages")
    return ctypes.byref(p.c())


def _rows(t, what, p: PagedParams, pages: Pages, T, heads):
    """The C view of a [rows][T][heads][128] tensor of the cache's type, any strides but adjacent values."""
    if t.dtype is not (_fp16 if p.half else _bf16) or t.get_device() != pages.index:
        raise ValueError(f"{what} must be a CUDA tensor of {'fp16' if p.half else 'bf16'} on the pool's device")
    if t.shape != (pages.rows, T, heads, 128):
        raise ValueError(f"{what} must be [{pages.rows}][{T}][{heads}][128], got {list(t.shape)}")
    sb, st, sh, sd = t.stride()
    if sd != 1:
        raise ValueError(f"{what} must have adjacent values in its last axis")
    return _Rows(t.data_ptr(), sb, st, sh)


def _tokens(t, what):
    if t.dim() != 4:
        raise ValueError(f"{what} must be [rows][T][heads][128], got {list(t.shape)}")
    return t.shape[1]


def _workspace(ws, pages, stream, size, *args):
    """ws, its address and its bytes; one of size(*args) bytes from torch's allocator, the stream's own, for None."""
    if ws is None:
        # asked for on the stream that uses it: the allocator hands a block that was given back to the same stream alone
        n = size(*args)
        if stream is not None and not hasattr(stream, "cuda_stream"):
            stream = _torch.cuda.ExternalStream(stream, device=pages.device)
        with nullcontext() if stream is None else _torch.cuda.stream(stream):
            ws = _torch.empty(n, dtype=_torch.uint8, device=pages.device)
    elif ws.get_device() != pages.index or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous CUDA tensor on the pool's device")
    return ws, ws.data_ptr(), ws.nbytes


def akv_paged_append(p: PagedParams, pages: Pages, K, V, n_new=None, layer: int = 0, stream=None):
    """K, V: [rows][T][n_kv_heads][128]; n_new: CUDA int32 [rows] (None: T each).  lens is not advanced.  Pages with more
    than one holder are not written."""
    if _device() != pages.index:
        return _there(pages, akv_paged_append, p, pages, K, V, n_new, layer, stream)
    T = _tokens(K, "K")
    _check(_lib().akv_paged_append(_params(p, pages), pages.ref, layer, _rows(K, "K", p, pages, T, p.n_kv_heads),
                                   _rows(V, "V", p, pages, T, p.n_kv_heads), T,
                                   _ints(n_new, "n_new", pages.rows, pages.index), _stream(stream, pages)),
           "akv_paged_append")


def akv_paged_read(p: PagedParams, pages: Pages, K, V, start=None, layer: int = 0, stream=None):
    """Fills K, V [rows][T][n_kv_heads][128] (any strides, e.g. a transposed [rows][n_kv_heads][T][128]) with the
    tokens from start (CUDA int32 [rows], None: 0) on; tokens that a request does not hold are zeros."""
    if _device() != pages.index:
        return _there(pages, akv_paged_read, p, pages, K, V, start, layer, stream)
    T = _tokens(K, "K")
    _check(_lib().akv_paged_read(_params(p, pages), pages.ref, layer, _ints(start, "start", pages.rows, pages.index),
                                 _rows(K, "K", p, pages, T, p.n_kv_heads), _rows(V, "V", p, pages, T, p.n_kv_heads), T,
                                 _stream(stream, pages)), "akv_paged_read")


def akv_paged_attn_workspace_size(p: PagedParams, pages: Pages, T: int = 1, top: int = 0) -> int:
    n = _sz()
    _check(_lib().akv_paged_attn_workspace_size(_params(p, pages), pages.ref, T, top, ctypes.byref(n)),
           "akv_paged_attn_workspace_size")
    return n.value


def _match(sel: PageSelection, pages: Pages, T, heads):
    if sel.count.shape != (pages.rows, T, heads) or sel.pages.device != pages.device:
        raise ValueError(f"the selection must be for [{pages.rows}][{T}][{heads}], on the pool's device")


def akv_paged_attn(p: PagedParams, pages: Pages, q, out, lse=None, sel: PageSelection | None = None,
                   sm_scale: float = 1.0, layer: int = 0, ws=None, stream=None):
    """q, out: [rows][T][n_q_heads][128]; lse: optional contiguous fp32 [rows][T][n_q_heads].
    ws: CUDA workspace of akv_paged_attn_workspace_size bytes; when None, one is taken from torch's allocator."""
    if _device() != pages.index:
        return _there(pages, akv_paged_attn, p, pages, q, out, lse, sel, sm_scale, layer, ws, stream)
    T = _tokens(q, "q")
    L = _lib()
    if sel is not None:
        _match(sel, pages, T, p.n_kv_heads)
    if lse is not None and (lse.dtype is not _torch.float32 or lse.get_device() != pages.index or not lse.is_contiguous()
                            or lse.shape != (pages.rows, T, p.n_q_heads)):
        raise ValueError(f"lse must be a contiguous CUDA fp32 tensor [{pages.rows}][{T}][{p.n_q_heads}]")
    ws, at, n = _workspace(ws, pages, stream, akv_paged_attn_workspace_size, p, pages, T, 0 if sel is None else sel.top)
    _check(L.akv_paged_attn(_params(p, pages), pages.ref, layer, _rows(q, "q", p, pages, T, p.n_q_heads),
                            _rows(out, "out", p, pages, T, p.n_q_heads), None if lse is None else lse.data_ptr(), T,
                            sm_scale, None if sel is None else sel.ref, at, n, _stream(stream, pages)), "akv_paged_attn")


def akv_paged_select_workspace_size(p: PagedParams, pages: Pages, T: int = 1) -> int:
    n = _sz()
    _check(_lib().akv_paged_select_workspace_size(_params(p, pages), pages.ref, T, ctypes.byref(n)),
           "akv_paged_select_workspace_size")
    return n.value


def akv_paged_select(p: PagedParams, pages: Pages, q, sel: PageSelection, sink: int = 1, recent: int = 1,
                     layer: int = 0, ws=None, stream=None):
    """q: [rows][T][n_q_heads][128]; fills sel.  ws as in akv_paged_attn, of akv_paged_select_workspace_size bytes."""
    if _device() != pages.index:
        return _there(pages, akv_paged_select, p, pages, q, sel, sink, recent, layer, ws, stream)
    T = _tokens(q, "q")
    L = _lib()
    _match(sel, pages, T, p.n_kv_heads)
    ws, at, n = _workspace(ws, pages, stream, akv_paged_select_workspace_size, p, pages, T)
    _check(L.akv_paged_select(_params(p, pages), pages.ref, layer, _rows(q, "q", p, pages, T, p.n_q_heads), T, sink, recent,
                              sel.ref, at, n, _stream(stream, pages)), "akv_paged_select")


def _shared(share: PageShare, pages: Pages):
    if share.rows != pages.rows or share.index != pages.index:
        raise ValueError(f"share must be for {pages.rows} rows, on the pool's device")
    return share.ref


def akv_pages_share(p: PagedParams, pages: Pages, share: PageShare, ws=None, stream=None):
    """Fills share: which rows begin with the same pages.  Once a step, for all layers.  ws as in akv_pages_reserve."""
    if _device() != pages.index:
        return _there(pages, akv_pages_share, p, pages, share, ws, stream)
    L = _lib()
    ref = _shared(share, pages)
    ws, at, n = _workspace(ws, pages, stream, akv_pages_workspace_size, pages)
    _check(L.akv_pages_share(_params(p, pages), pages.ref, ref, at, n, _stream(stream, pages)), "akv_pages_share")


def akv_paged_attn_shared_workspace_size(p: PagedParams, pages: Pages, T: int = 1) -> int:
    n = _sz()
    _check(_lib().akv_paged_attn_shared_workspace_size(_params(p, pages), pages.ref, T, ctypes.byref(n)),
           "akv_paged_attn_shared_workspace_size")
    return n.value


def _lse(lse, p: PagedParams, pages: Pages, T):
    if (lse.dtype is not _torch.float32 or lse.get_device() != pages.index or not lse.is_contiguous()
            or lse.shape != (pages.rows, T, p.n_q_heads)):
        raise ValueError(f"lse must be a contiguous CUDA fp32 tensor [{pages.rows}][{T}][{p.n_q_heads}]")
    return lse.data_ptr()


def akv_paged_attn_shared(p: PagedParams, pages: Pages, q, out, share: PageShare, lse=None, sm_scale: float = 1.0,
                          layer: int = 0, ws=None, stream=None):
    """akv_paged_attn over rows that share pages (share of akv_pages_share): those are read once for all, where that pays.
    Without forked rows akv_paged_attn is the faster call.
    ws as there, of akv_paged_attn_shared_workspace_size bytes."""
    if _device() != pages.index:
        return _there(pages, akv_paged_attn_shared, p, pages, q, out, share, lse, sm_scale, layer, ws, stream)
    T = _tokens(q, "q")
    L = _lib()
    ref = _shared(share, pages)
    lse = None if lse is None else _lse(lse, p, pages, T)
    ws, at, n = _workspace(ws, pages, stream, akv_paged_attn_shared_workspace_size, p, pages, T)
    _check(L.akv_paged_attn_shared(_params(p, pages), pages.ref, layer, _rows(q, "q", p, pages, T, p.n_q_heads),
                                   _rows(out, "out", p, pages, T, p.n_q_heads), lse, T, sm_scale, ref, at, n,
                                   _stream(stream, pages)), "akv_paged_attn_shared")


def _scores(t, what, p: PagedParams, pages: Pages):
    """The C view of an fp32 [rows][n_kv_heads][cap] tensor with adjacent numbers in its last axis."""
    if t.dtype is not _torch.float32 or t.get_device() != pages.index:
        raise ValueError(f"{what} must be a CUDA fp32 tensor on the pool's device")
    if t.dim() != 3 or t.shape[:2] != (pages.rows, p.n_kv_heads):
        raise ValueError(f"{what} must be [{pages.rows}][{p.n_kv_heads}][cap], got {list(t.shape)}")
    sb, sh, si = t.stride()
    if si != 1 and t.shape[2] > 1:
        raise ValueError(f"{what} must have adjacent numbers in its last axis")
    return _Scores(t.data_ptr(), sb, sh, min(t.shape[2], 2**31 - 1))


def akv_paged_weights_workspace_size(p: PagedParams, pages: Pages, T: int = 1) -> int:
    n = _sz()
    _check(_lib().akv_paged_weights_workspace_size(_params(p, pages), pages.ref, T, ctypes.byref(n)),
           "akv_paged_weights_workspace_size")
    return n.value


def akv_paged_weights(p: PagedParams, pages: Pages, q, lse, now, was=None, decay: float = 1.0, sm_scale: float = 1.0,
                      layer: int = 0, ws=None, stream=None):
    """now = decay was + the attention weights of the last T query tokens.  q: [rows][T][n_q_heads][128], lse of
    akv_paged_attn; now, was: fp32 [rows][n_kv_heads][cap], was None (zeros), now itself or apart from it.  A new token begins
    with what stands at its place: set that to 0, also where a place is used again.  ws as there, of
    akv_paged_weights_workspace_size bytes."""
    if _device() != pages.index:
        return _there(pages, akv_paged_weights, p, pages, q, lse, now, was, decay, sm_scale, layer, ws, stream)
    T = _tokens(q, "q")
    L = _lib()
    ws, at, n = _workspace(ws, pages, stream, akv_paged_weights_workspace_size, p, pages, T)
    _check(L.akv_paged_weights(_params(p, pages), pages.ref, layer, _rows(q, "q", p, pages, T, p.n_q_heads),
                               _lse(lse, p, pages, T), T, sm_scale, decay,
                               None if was is None else _scores(was, "was", p, pages), _scores(now, "now", p, pages),
                               at, n, _stream(stream, pages)), "akv_paged_weights")


def akv_paged_evict(p: PagedParams, pages: Pages, src, dst, scores, kept: KeptTokens, keep=None, sink: int = 0,
                    recent: int = 0, layer: int = 0, stream=None):
    """Row dst[i] gets the tokens that row src[i] keeps by their scores (CUDA int32 [n]; the same row: in place).  scores: fp32
    [rows][n_kv_heads][cap]; keep: CUDA int32 [n] (None: kept.top each); fills kept.  lens is not changed, nor are
    the scores behind what is kept."""
    if _device() != pages.index:
        return _there(pages, akv_paged_evict, p, pages, src, dst, scores, kept, keep, sink, recent, layer, stream)
    a, b, n = _pair(src, dst, pages)
    if tuple(kept.tokens.shape[:2]) != (n, p.n_kv_heads) or kept.tokens.device != pages.device:
        raise ValueError(f"kept must be for [{n}][{p.n_kv_heads}], on the pool's device")
    _check(_lib().akv_paged_evict(_params(p, pages), pages.ref, layer, a, b, n, _scores(scores, "scores", p, pages),
                                  _ints(keep, "keep", n, pages.index), sink, recent, kept.ref, _stream(stream, pages)),
           "akv_paged_evict")


def akv_pages_trim(p: PagedParams, pages: Pages, rows, stream=None):
    """Rows (CUDA int32) give up the pages behind their length."""
    if _device() != pages.index:
        return _there(pages, akv_pages_trim, p, pages, rows, stream)
    _check(_lib().akv_pages_trim(_params(p, pages), pages.ref, _ints(rows, "rows", None, pages.index), rows.numel(),
                                 _stream(stream, pages)), "akv_pages_trim")


def _pair(src, dst, pages):
    n = src.numel()
    return _ints(src, "src", None, pages.index), _ints(dst, "dst", n, pages.index), n


def akv_pages_copy(p: PagedParams, pages: Pages, src, dst, stream=None):
    """Copies page src[i] to page dst[i] in every layer (CUDA int32)."""
    if _device() != pages.index:
        return _there(pages, akv_pages_copy, p, pages, src, dst, stream)
    a, b, n = _pair(src, dst, pages)
    _check(_lib().akv_pages_copy(_params(p, pages), pages.ref, a, b, n, _stream(stream, pages)), "akv_pages_copy")


def akv_pages_fork(p: PagedParams, pages: Pages, src, dst, stream=None):
    """Row dst[i] becomes a second holder of row src[i]'s pages (CUDA int32)."""
    if _device() != pages.index:
        return _there(pages, akv_pages_fork, p, pages, src, dst, stream)
    a, b, n = _pair(src, dst, pages)
    _check(_lib().akv_pages_fork(_params(p, pages), pages.ref, a, b, n, _stream(stream, pages)), "akv_pages_fork")


def akv_pages_workspace_size(pages: Pages) -> int:
    n = _sz()
    _check(_lib().akv_pages_workspace_size(pages.pref, pages.ref, ctypes.byref(n)), "akv_pages_workspace_size")
    return n.value


def akv_pages_reserve(p: PagedParams, pages: Pages, n_new, missing, ws=None, stream=None):
    """Pages for each row's next n_new tokens (CUDA int32 [rows]); missing: CUDA int32 [1]."""
    if _device() != pages.index:
        return _there(pages, akv_pages_reserve, p, pages, n_new, missing, ws, stream)
    ws, at, n = _workspace(ws, pages, stream, akv_pages_workspace_size, pages)
    _check(_lib().akv_pages_reserve(_params(p, pages), pages.ref, _ints(n_new, "n_new", pages.rows, pages.index),
                                    _ints(missing, "missing", 1, pages.index), at, n, _stream(stream, pages)), "akv_pages_reserve")


def akv_pages_free(p: PagedParams, pages: Pages, rows, stream=None):
    """Rows (CUDA int32) give up their pages."""
    if _device() != pages.index:
        return _there(pages, akv_pages_free, p, pages, rows, stream)
    _check(_lib().akv_pages_free(_params(p, pages), pages.ref, _ints(rows, "rows", None, pages.index), rows.numel(),
                                 _stream(stream, pages)), "akv_pages_free")


def akv_pages_compact(p: PagedParams, pages: Pages, n_live, ws=None, stream=None):
    """Moves live pages to the front of the pool; n_live: CUDA int32 [1]."""
    if _device() != pages.index:
        return _there(pages, akv_pages_compact, p, pages, n_live, ws, stream)
    ws, at, n = _workspace(ws, pages, stream, akv_pages_workspace_size, pages)
    _check(_lib().akv_pages_compact(_params(p, pages), pages.ref, _ints(n_live, "n_live", 1, pages.index), at, n,
                                    _stream(stream, pages)), "akv_pages_compact")
