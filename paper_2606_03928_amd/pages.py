"""The paged KV cache of libvase.so (``include/vase_page.h``).

A :class:`PageCache` holds the K and V rows of S sequence slots in a pool of pages that
sequences take, share and give up, where the static cache of :mod:`.vase` holds K + B rows
for each whether used or not.  Argument marshalling only, as in :mod:`.vase`: the work
runs in the library's HIP kernels on the current stream, nothing synchronises, and
errors are ``ValueError`` (arguments) or :class:`.vase.VaseError` (the library).

  * :meth:`PageCache.attn`     -- attention of each slot's newest rows (a token, a chunk)
  * :meth:`PageCache.write`    -- the rows of new tokens into their slots
  * :meth:`PageCache.resize`   -- slots truncated and grown: pages freed, taken, copied
  * :meth:`PageCache.fork`     -- slots that begin as another's, on the same pages
  * :meth:`PageCache.compact`  -- the survivors of an eviction round (``vase.select``'s map)

A step of serving: ``resize`` to the new lengths, ``write`` and ``attn`` layer by layer
(``cache.heads(first, count)`` is one layer's view, made once and kept); every B steps a
round: a survivor map from ``vase.score`` and ``vase.select``, then ``compact`` for all heads.
``vase.score`` takes rows that lie together: with pages of K + B rows and one page to a
slot, ``cache.k.view(-1, K + B, d)`` is the static cache that it and ``vase.Round`` take.  On
smaller pages the rows are first gathered through the table into such a cache.

Data that only the device knows (lengths, page numbers) is checked there: a call that meets
a bad value, or too few free pages, ORs a ``STATUS_PAGE_*`` bit into ``status`` (an int32
device tensor given to the constructor or to the call).
"""
from __future__ import annotations

import ctypes
import threading
from typing import Optional

import torch

from . import vase
from .vase import _ptr, _require, _stream_ptr

STATUS_PAGE_FULL, STATUS_PAGE_BAD = 16, 32
OP_PAGE_ATTN, OP_PAGE_RESIZE, OP_PAGE_COMPACT = 0, 1, 2
MAX_ROWS = 1 << 29        # M * page


class _Pages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("ref", ctypes.c_void_p),
                ("table", ctypes.c_void_p), ("len", ctypes.c_void_p), ("page_stride", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("H", ctypes.c_int32),
                ("page", ctypes.c_int32), ("d", ctypes.c_int32), ("S", ctypes.c_int32),
                ("M", ctypes.c_int32)]


_lock = threading.Lock()
_ready = None


def load() -> ctypes.CDLL:
    """libvase.so with the paged cache's entry points."""
    global _ready
    if _ready is not None:
        return _ready
    lib = vase.load()
    with _lock:
        C, P, I, L, SZ = (ctypes.POINTER(_Pages), ctypes.c_void_p, ctypes.c_int, ctypes.c_int64,
                          ctypes.c_size_t)
        lib.vase_page_workspace_bytes.argtypes = [I, C, I, I, I, I]
        lib.vase_page_workspace_bytes.restype = SZ
        lib.vase_page_attn.argtypes = [C, P, L, P, I, I, I, I, I, P, P, P, SZ, P, P]
        lib.vase_page_write.argtypes = [C, P, P, L, P, I, P, P]
        lib.vase_page_resize.argtypes = [C, P, P, SZ, P, P]
        lib.vase_page_fork.argtypes = [C, P, P, P]
        lib.vase_page_compact.argtypes = [C, P, P, I, I, P, SZ, P, P]
        for name in ("attn", "write", "resize", "fork", "compact"):
            getattr(lib, "vase_page_" + name).restype = I
        _ready = lib
    return lib


def _ints(t: torch.Tensor, shape, device, name: str) -> int:
    if not (t.dtype is torch.int32 and t.shape == shape and t.device == device and t.is_contiguous()):
        raise ValueError("%s must be a contiguous int32 tensor %s on the cache's device"
                         % (name, list(shape)))
    return t.data_ptr()


def _token_rows(t: torch.Tensor, heads: Optional[int], like: "PageCache", name: str) -> int:
    """The token stride of [T, heads, d] rows whose heads and elements are contiguous."""
    if not (t.dim() == 3 and t.dtype is like.dtype and t.device == like.device):
        raise ValueError("%s must be [T, heads, d] of the cache's dtype, on its device" % name)
    T, H, d = t.shape
    stride, head, one = t.stride()
    least = H * d
    if T <= 1:
        stride = least          # of a single token (or none) the stride says nothing
    if d != like.d or (heads is not None and H != heads):
        raise ValueError("%s must be [T, heads, d] of the cache's heads and row length" % name)
    if one != 1 or (head != d and H != 1) or stride < least:
        raise ValueError("%s must have contiguous heads, and tokens that do not overlap" % name)
    return stride


class PageCache:
    """K and V pools [n_pages, H, page, d] (bf16 or fp32; a page's heads contiguous, any stride
    from page to page, the same in both), ref [n_pages], table [S, M] and length [S] int32,
    all on one device and all the caller's: a page is free where ref is 0, a slot where
    length is.  The tensors are used in place and kept alive."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, ref: torch.Tensor, table: torch.Tensor,
                 length: torch.Tensor, status: Optional[torch.Tensor] = None):
        for t, n in ((k, "k"), (v, "v")):
            _require(t.is_cuda, "%s must be a device tensor" % n)
            _require(t.dim() == 4, "%s must be [n_pages, H, page, d]" % n)
        P, H, page, d = k.shape
        _require(v.shape == k.shape and v.dtype == k.dtype and v.device == k.device,
                 "k and v must have one shape and dtype, on one device")
        for t, n in ((k, "k"), (v, "v")):
            _require(t.stride(3) == 1 and t.stride(2) == d and (H == 1 or t.stride(1) == page * d),
                     "%s: the heads of a page must be contiguous" % n)
        stride = [t.stride(0) if P > 1 else H * page * d for t in (k, v)]
        _require(stride[0] == stride[1], "k and v must have one stride from page to page")
        _require(page % 16 == 0 and page >= 16, "page must be a multiple of 16 rows")
        _require(table.dim() == 2 and length.dim() == 1, "table must be [S, M], length [S]")
        S, M = table.shape
        dev = k.device
        self.k, self.v, self.ref, self.table, self.length = k, v, ref, table, length
        self.S, self.M, self.n_pages, self.H, self.page, self.d = S, M, P, H, page, d
        self.device, self.dtype = dev, k.dtype
        self.status = status
        self._status_word = vase._status_ptr(status, dev)
        self._c = _Pages(_ptr(k), _ptr(v), _ints(ref, (P,), dev, "ref"), _ints(table, (S, M), dev, "table"),
                         _ints(length, (S,), dev, "length"), stride[0], vase.dtype_code(k.dtype), P, H,
                         page, d, S, M)
        self._need = {}          # workspace bytes by operation and sizes
        self._state_ws = None    # of resize and compact, made by the first of them
        self._lib = load()
        self._by = ctypes.byref(self._c)

    @classmethod
    def new(cls, n_pages: int, H: int, page: int, d: int, S: int, M: int,
            dtype: torch.dtype = torch.bfloat16, device="cuda", status: bool = True) -> "PageCache":
        """An empty cache of its own pools (and a status word, zero)."""
        def ints(*shape):
            return torch.zeros(shape, dtype=torch.int32, device=device)
        k = torch.empty((n_pages, H, page, d), dtype=dtype, device=device)
        return cls(k, torch.empty_like(k), ints(n_pages), ints(S, M) - 1, ints(S),
                   status=ints(1) if status else None)

    def heads(self, first: int, count: int) -> "PageCache":
        """The same cache with `count` heads from `first` on (a layer's), for write and attn.  To be
        kept for as long as the cache: making it checks all of the cache's tensors anew."""
        _require(0 <= first and 1 <= count and first + count <= self.H, "heads out of range")
        return _Heads(self, first, count)

    # -- helpers -----------------------------------------------------------------------

    def _bytes(self, op: int, T: int = 0, G: int = 0, max_new: int = 0, max_len: int = 0) -> int:
        key = (op, T, G, max_new, max_len)
        n = self._need.get(key)
        if n is None:
            if len(self._need) >= 256:
                self._need.clear()
            n = self._need[key] = int(self._lib.vase_page_workspace_bytes(
                op, self._by, T, G, max_new, max_len))
        return n

    def attn_workspace_bytes(self, T: int, G: int, max_new: int, max_len: Optional[int] = None) -> int:
        """Bytes that attn takes as ws for these sizes (0: none)."""
        # not by way of _bytes, where a float finds what an equal whole number has left
        return int(self._lib.vase_page_workspace_bytes(
            OP_PAGE_ATTN, self._by, T, G, max_new, self.M * self.page if max_len is None else max_len))

    def state_workspace_bytes(self) -> int:
        """Bytes that resize and compact take as ws."""
        return max(self._bytes(OP_PAGE_RESIZE), self._bytes(OP_PAGE_COMPACT))

    def _scratch(self, nbytes: int, stream) -> torch.Tensor:
        """Memory of the stream that will use it: what lay there before was that stream's."""
        if stream is None:
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        with torch.cuda.stream(stream):
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device)

    @staticmethod
    def _capturing(stream) -> bool:
        if stream is None:
            return torch.cuda.is_current_stream_capturing()
        with torch.cuda.stream(stream):
            return torch.cuda.is_current_stream_capturing()

    def _ws(self, ws, nbytes: int, stream):
        """(pointer, bytes, tensor) of the given workspace or a new one."""
        if ws is None:
            if nbytes == 0:
                return None, 0, None
            ws = self._scratch(nbytes, stream)
            return ws.data_ptr(), nbytes, ws
        _require(ws.is_cuda and ws.device == self.device and ws.is_contiguous(),
                 "ws must be a contiguous tensor on the cache's device")
        have = ws.numel() * ws.element_size()
        _require(have >= nbytes, "workspace too small")
        return ws.data_ptr(), have, ws

    def _state(self, ws, op: int, stream):
        """As _ws, for resize and compact: by default the cache's own, as calls that change one
        cache follow each other in any case.  A captured call takes one of its graph's."""
        if ws is None and not self._capturing(stream):
            ws = self._state_ws
            if ws is None:
                ws = self._state_ws = self._scratch(self.state_workspace_bytes(), stream)
                self._state_home = _stream_ptr(self.device, stream)
            if _stream_ptr(self.device, stream) != self._state_home:
                ws.record_stream(stream if stream is not None else torch.cuda.current_stream(self.device))
            return ws.data_ptr(), ws.numel(), ws
        return self._ws(ws, self._bytes(op), stream)

    def _status(self, status):
        return self._status_word if status is None else vase._status_ptr(status, self.device)

    def _call(self, f, name: str, *args):
        if torch.cuda.current_device() == self.device.index:
            rc = f(self._by, *args)
        else:
            with torch.cuda.device(self.device):
                rc = f(self._by, *args)
        if rc != vase.OK:
            raise vase.VaseError(name, rc)

    # -- operators ---------------------------------------------------------------------

    def attn(self, q: torch.Tensor, cu: torch.Tensor, max_new: int, max_len: Optional[int] = None,
             causal: bool = True, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
             ws: Optional[torch.Tensor] = None, stream=None,
             status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of the batch's tokens q [T, H * G, d] over their slots (vase_page_attn).

        cu [S + 1] int32: tokens cu[s] .. cu[s + 1] are slot s's newest rows, already
        written.  max_new: the most tokens of a slot; max_len: the longest slot's rows (for
        the split of the work; by default what the table can hold).  q may be a part
        of a wider tensor: any stride from token to token.  lse [T, H * G] float32 takes
        the rows' log-sum-exp.  Returns out [T, H * G, d]; the tokens from cu[S] on, if
        any, are left as they were (zero in an out made here, by a launch of its own)."""
        stride = _token_rows(q, None, self, "q")
        T, HG, d = q.shape
        G, rest = divmod(HG, self.H)
        if rest or G < 1:
            raise ValueError("q must have G query heads for each of the cache's heads")
        if max_len is None:
            max_len = self.M * self.page
        cup = _ints(cu, (self.S + 1,), self.device, "cu")
        if out is None:
            out = torch.zeros((T, HG, self.d), dtype=q.dtype, device=self.device)
            if stream is not None:
                # the zeros are written on the current stream
                stream.wait_stream(torch.cuda.current_stream(self.device))
                out.record_stream(stream)
        elif not (out.shape == q.shape and out.dtype is q.dtype and out.device == self.device
                  and out.is_contiguous()):
            raise ValueError("out must be contiguous, like q")
        lp = None
        if lse is not None:
            lp = lse.data_ptr()
            _require(lse.dtype == torch.float32 and tuple(lse.shape) == (T, HG) and lse.is_contiguous()
                     and lse.device == self.device, "lse must be contiguous float32 [T, H * G]")
        wp, wn, ws = self._ws(ws, self._bytes(OP_PAGE_ATTN, T, G, max_new, max_len) if T else 0, stream)
        self._call(self._lib.vase_page_attn, "vase_page_attn", q.data_ptr(), stride, cup, T, G, max_new,
                   max_len, 1 if causal else 0, out.data_ptr(), lp, wp, wn, self._status(status),
                   _stream_ptr(self.device, stream))
        return out

    def write(self, k_new: torch.Tensor, v_new: torch.Tensor, cu: torch.Tensor, stream=None,
              status: Optional[torch.Tensor] = None) -> None:
        """The tokens' rows k_new, v_new [T, H, d] into the last rows of their slots: token i of
        slot s's n into row length[s] - n + i (vase_page_write).  Both may be parts of wider
        tensors with one stride from token to token."""
        a = _token_rows(k_new, self.H, self, "k_new")
        T = k_new.shape[0]
        if a != _token_rows(v_new, self.H, self, "v_new") or v_new.shape[0] != T:
            raise ValueError("k_new and v_new must have one shape and stride")
        self._call(self._lib.vase_page_write, "vase_page_write", k_new.data_ptr(), v_new.data_ptr(), a,
                   _ints(cu, (self.S + 1,), self.device, "cu"), T,
                   self._status(status), _stream_ptr(self.device, stream))

    def resize(self, new_len: torch.Tensor, ws: Optional[torch.Tensor] = None, stream=None,
               status: Optional[torch.Tensor] = None) -> None:
        """The slots' lengths become new_len [S] int32 (negative: left alone): pages are given
        up, taken (the lowest free ones), and copied where a slot grows within a page that it
        shares.  All or nothing: STATUS_PAGE_FULL with too few free pages (vase_page_resize)."""
        p = _ints(new_len, (self.S,), self.device, "new_len")
        wp, wn, ws = self._state(ws, OP_PAGE_RESIZE, stream)
        self._call(self._lib.vase_page_resize, "vase_page_resize", p, wp, wn, self._status(status),
                   _stream_ptr(self.device, stream))

    def fork(self, parent: torch.Tensor, stream=None, status: Optional[torch.Tensor] = None) -> None:
        """Each free slot s with parent[s] >= 0 (parent [S] int32) begins as that slot: its
        rows, on the same pages (vase_page_fork)."""
        self._call(self._lib.vase_page_fork, "vase_page_fork", _ints(parent, (self.S,), self.device, "parent"),
                   self._status(status), _stream_ptr(self.device, stream))

    def compact(self, map: torch.Tensor, src: torch.Tensor, ws: Optional[torch.Tensor] = None,
                stream=None, status: Optional[torch.Tensor] = None) -> None:
        """Each slot s with map[s] >= 0 (map [S] int32) keeps the K rows src[map[s]][h] of head
        h, in order (src [n_map, H, K] int32, survivor maps as vase.select's); the pages behind
        them are given up, and shared pages left to the others (vase_page_compact)."""
        _require(src.dim() == 3 and src.shape[1] == self.H, "src must be [n_map, H, K]")
        n_map, K = int(src.shape[0]), int(src.shape[2])
        sp = _ints(src, src.shape, self.device, "src")
        mp = _ints(map, (self.S,), self.device, "map")
        wp, wn, ws = self._state(ws, OP_PAGE_COMPACT, stream)
        self._call(self._lib.vase_page_compact, "vase_page_compact", mp, sp, n_map, K, wp, wn, self._status(status),
                   _stream_ptr(self.device, stream))


class _Heads(PageCache):
    """Some of a cache's heads: rows are written and attended to, lengths and pages are the
    whole cache's to change."""

    def __init__(self, cache: PageCache, first: int, count: int):
        super().__init__(cache.k[:, first:first + count], cache.v[:, first:first + count], cache.ref,
                         cache.table, cache.length, cache.status)

    def resize(self, *args, **kw):
        raise ValueError("resize takes all heads of the cache")

    def compact(self, *args, **kw):
        raise ValueError("compact takes all heads of the cache")

    def fork(self, *args, **kw):
        raise ValueError("fork takes all heads of the cache")
