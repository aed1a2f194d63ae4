"""ctypes binding of the paged cache's entry points of libpgxgo.so; names follow include/pgxcache.h (pgxcache_<name> -> PagedCache.<name>)."""
import ctypes as C
import operator

import torch

from . import binding
from .binding import PgxGoError, _address, _need, _ptr, lib as _golib

TYPES = {torch.float16: 1, torch.bfloat16: 2}
HEAD_DIMS = (32, 64, 96, 128, 256)
NO_PAGES, FULL, BAD_ENTRY = 1, 2, 255
_ready = False
_fast = None   # as in binding.py


class _Opts(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("slots", "pages", "width", "page_size", "layers", "kv_heads", "head_dim", "type")] + [("stream", C.c_void_p)]


def lib():
    """The shared library with the pgxcache_* prototypes declared; raises if it has not been built (no fallback)."""
    global _ready, _fast
    L = _golib()
    if not _ready:
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.pgxcache_work_bytes.restype = C.c_size_t
        L.pgxcache_work_bytes.argtypes = [C.POINTER(_Opts)]
        L.pgxcache_init.argtypes = [C.POINTER(vp), C.POINTER(_Opts), vp, vp, vp, vp, vp, C.c_size_t]
        L.pgxcache_destroy.argtypes = [vp]
        L.pgxcache_rescan.argtypes = [vp]
        L.pgxcache_advance.argtypes = [vp, i32, vp, vp, i32, vp]
        L.pgxcache_write.argtypes = [vp, i32, i32, vp, i32, vp, i64, i64, i64, vp, i64, i64, i64]
        L.pgxcache_attend.argtypes = [vp, i32, i32, vp, i32, vp, i64, i64, vp, i64, i64, vp, i64, i64, C.c_float, vp, i64, i64, vp]
        L.pgxcache_fork.argtypes = [vp, i32, vp, vp, vp]
        L.pgxcache_free.argtypes = [vp, i32, vp]
        L.pgxcache_compact.argtypes = [vp, vp]
        L.pgxcache_strerror.restype = C.c_char_p
        L.pgxcache_strerror.argtypes = [C.c_int]
        L.pgxcache_last_hip_error.restype = C.c_int
        _fast = binding._fast
        _ready = True
    return L


def _check(rc, what):
    if rc != 0:
        L = lib()
        raise PgxGoError(f"{what}: {L.pgxcache_strerror(rc).decode()} (code {rc}, hip error {L.pgxcache_last_hip_error()})")


def _whole(x, name):
    """a whole number that the entry points' 32 bits hold (ctypes would cut it off)"""
    try:
        n = operator.index(x)
    except TypeError:
        n = None
    if n is None or not -2 ** 31 <= n < 2 ** 31:
        raise PgxGoError(f"{name}: expected a whole number of 32 bits, got {x!r}")
    return n


class PagedCache:
    """Keys and values of a pool of game states, in pages that copies of a state share (include/pgxcache.h).

    The memory is the caller's: kv [pages][layers][2][kv_heads][page_size][head_dim] in float16 or bfloat16, table int32 [slots][width],
    lengths int32 [slots], refs int32 [pages].  The handle takes them as they are (PagedCache.empty makes empty ones), so a cache
    is saved by copying the four and restored by making a handle on them; after writing to refs oneself, call rescan().
    All calls run on the stream that was current when the handle was made, and attend's new outputs belong to it, whichever stream is
    current: a program that works on another one has the two wait for each other, as for tensors of any other stream."""

    def __init__(self, kv, table, lengths, refs):
        L = lib()
        if not isinstance(kv, torch.Tensor) or kv.dtype not in TYPES or kv.dim() != 6 or kv.shape[2] != 2 or not kv.is_cuda or not kv.is_contiguous():
            raise PgxGoError("kv: expected a contiguous cuda tensor [pages][layers][2][kv_heads][page_size][head_dim] of float16 or bfloat16")
        pages, self.layers, _, self.kv_heads, self.page_size, self.head_dim = kv.shape
        if getattr(table, "ndim", 0) != 2:
            raise PgxGoError("table: expected int32 [slots][width]")
        self.slots, self.width = table.shape
        _need(table, torch.int32, (self.slots, self.width), "table")
        _need(lengths, torch.int32, (self.slots,), "lengths")
        _need(refs, torch.int32, (pages,), "refs")
        if any(t.device != kv.device for t in (table, lengths, refs)):
            raise PgxGoError(f"table, lengths and refs have to be on {kv.device}, as kv is")
        self.pages, self.dtype, self.device = pages, kv.dtype, kv.device
        self.kv, self.table, self.lengths, self.refs = kv, table, lengths, refs
        with torch.cuda.device(self.device):
            self._stream = torch.cuda.current_stream(self.device)
            opts = _Opts(self.slots, pages, self.width, self.page_size, self.layers, self.kv_heads, self.head_dim, TYPES[kv.dtype], self._stream.cuda_stream)
            nbytes = L.pgxcache_work_bytes(C.byref(opts))
            if nbytes == 0:
                raise PgxGoError(f"cache: pages of a power of two from 16 to 1024 tokens, heads of {HEAD_DIMS} elements; got {self.page_size} and {self.head_dim}")
            self._work = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            h = C.c_void_p()
            _check(L.pgxcache_init(C.byref(h), C.byref(opts), _ptr(kv), _ptr(table), _ptr(lengths), _ptr(refs), _ptr(self._work), nbytes), "pgxcache_init")
        self._h, self._destroy = h, L.pgxcache_destroy
        if _fast is not None:
            self._calls = {n: _address(getattr(L, "pgxcache_" + n)) for n in ("advance", "write", "attend", "fork", "free")}
            self._shape = (self.slots, self.kv_heads, self.head_dim, TYPES[self.dtype], self.device.index, self._stream.stream_id)
        self._scale = self.head_dim ** -0.5

    @classmethod
    def empty(cls, slots, pages, max_length, layers, kv_heads, head_dim, page_size=16, dtype=torch.bfloat16, device="cuda:0"):
        """An empty cache of slots that hold up to max_length tokens each (rounded up to whole pages)."""
        kv = torch.empty((pages, layers, 2, kv_heads, page_size, head_dim), dtype=dtype, device=device)
        table = torch.full((slots, (max_length + page_size - 1) // page_size), -1, dtype=torch.int32, device=device)
        zeros = lambda n: torch.zeros(n, dtype=torch.int32, device=device)  # noqa: E731
        return cls(kv, table, zeros(slots), zeros(pages))

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h:
            self._destroy(h)   # (module globals may be gone when the interpreter shuts down)

    def _list(self, slots, name="slots"):
        """number of entries, pointer"""
        if slots is None:
            return self.slots, None
        if not isinstance(slots, torch.Tensor) or slots.dim() != 1:
            raise PgxGoError(f"{name}: expected int32 [n]")
        n = slots.shape[0]
        if n > self.slots:
            raise PgxGoError(f"{name}: {n} entries for {self.slots} slots")
        self._own(slots, torch.int32, (n,), name)
        return n, slots.data_ptr()

    def _own(self, t, dtype, shape, name):
        """a contiguous tensor on the cache's device"""
        if not isinstance(t, torch.Tensor) or t.device != self.device:
            raise PgxGoError(f"{name}: expected a tensor on {self.device}, as the cache is, got {t.device if isinstance(t, torch.Tensor) else type(t).__name__}")
        return _need(t, dtype, shape, name)

    def _status(self, status, n):
        return None if status is None else self._own(status, torch.uint8, (n,), "status").data_ptr()

    def _heads(self, t, shape, name):
        """pointer of a tensor of the cache's type whose last dimension is dense"""
        if (not isinstance(t, torch.Tensor) or t.dtype is not self.dtype or t.device != self.device or t.shape != shape
                or (t.stride(-1) != 1 and t.numel() > 0)):
            got = f"{t.dtype} {tuple(t.shape)} of strides {t.stride()} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
            raise PgxGoError(f"{name}: expected {self.dtype} tensor of shape {tuple(shape)} on {self.device} with a dense last dimension, got {got}")
        return t.data_ptr()

    def rescan(self):
        _check(lib().pgxcache_rescan(self._h), "pgxcache_rescan")

    def advance(self, slots=None, counts=1, status=None):
        """Room for counts (a number, or int32 [n]) more tokens in each of the slots (int32 [n], pairwise distinct; None: all)."""
        if _fast is not None:
            rc = _fast.cache_advance(self._calls["advance"], self._h.value, self._shape, slots, counts, status)
            if rc == 0: return
            if rc is not None: _check(rc, "pgxcache_advance")
        n, p = self._list(slots)
        each = isinstance(counts, torch.Tensor)
        if each: self._own(counts, torch.int32, (n,), "counts")
        elif not 0 <= _whole(counts, "counts") < 2 ** 31: raise PgxGoError(f"counts: 0 or more tokens, got {counts}")
        _check(lib().pgxcache_advance(self._h, n, p, _ptr(counts) if each else None, 0 if each else operator.index(counts), self._status(status, n)), "pgxcache_advance")

    def write(self, layer, k, v, slots=None):
        """Keys and values of the tokens that the slots' last advance made room for: [n][kv_heads][head_dim], or [n][tokens][kv_heads][head_dim]
        of which a slot takes as many as it has room for."""
        if _fast is not None:
            rc = _fast.cache_write(self._calls["write"], self._h.value, self._shape, layer, k, v, slots)
            if rc == 0: return
            if rc is not None: _check(rc, "pgxcache_write")
        n, p = self._list(slots)
        many = getattr(k, "ndim", 0) == 4
        tokens = k.shape[1] if many else 1
        shape = (n, tokens, self.kv_heads, self.head_dim) if many else (n, self.kv_heads, self.head_dim)
        kp, vp = self._heads(k, shape, "k"), self._heads(v, shape, "v")
        ks, vs = ((t.stride(0), t.stride(1) if many else 0, t.stride(-2)) for t in (k, v))
        _check(lib().pgxcache_write(self._h, _whole(layer, "layer"), n, p, tokens, kp, *ks, vp, *vs), "pgxcache_write")

    def attend(self, layer, q, slots=None, k=None, v=None, scale=None, out=None, lse=False):
        """Attention of one token per slot, q [n][heads][head_dim], over the slot's tokens; heads a multiple of kv_heads; scale: head_dim ** -0.5.
        k and v [n][kv_heads][head_dim] (both or neither): the newest token's, written to the cache on the way.  Returns out, or with
        lse (True, or a float32 [n][heads] tensor) out and the logarithms of the sums of exponentials."""
        scale = self._scale if scale is None else scale
        if _fast is not None:
            got = _fast.cache_attend(self._calls["attend"], self._h.value, self._shape, layer, q, slots, k, v, scale, out, lse)
            if type(got) is tuple: return got[0] if lse is False else got
            if got is not None: _check(got, "pgxcache_attend")
        n, p = self._list(slots)
        if getattr(q, "ndim", 0) != 3:
            raise PgxGoError("q: expected [n][heads][head_dim]")
        heads = q.shape[1]
        if heads < 1 or heads % self.kv_heads:
            raise PgxGoError(f"q: {heads} heads are no multiple of the cache's {self.kv_heads}")
        qp = self._heads(q, (n, heads, self.head_dim), "q")
        if (k is None) != (v is None):
            raise PgxGoError("k and v: both or neither")
        kp = vp = None
        ks = vs = (0, 0)
        if k is not None:
            shape = (n, self.kv_heads, self.head_dim)
            kp, vp = self._heads(k, shape, "k"), self._heads(v, shape, "v")
            ks, vs = k.stride()[:2], v.stride()[:2]
        with torch.cuda.stream(self._stream):   # new outputs belong to the stream that writes them
            if out is None: out = torch.empty((n, heads, self.head_dim), dtype=self.dtype, device=self.device)
            made = torch.empty((n, heads), dtype=torch.float32, device=self.device) if lse is True else None
        op = self._heads(out, (n, heads, self.head_dim), "out")
        if lse is True: lse = made
        elif lse is not False: self._own(lse, torch.float32, (n, heads), "lse")
        _check(lib().pgxcache_attend(self._h, _whole(layer, "layer"), n, p, heads, qp, *q.stride()[:2], kp, *ks, vp, *vs, float(scale), op, *out.stride()[:2],
                                     None if lse is False else lse.data_ptr()), "pgxcache_attend")
        return out if lse is False else (out, lse)

    def fork(self, src, dst, status=None):
        """slot[dst[i]] = slot[src[i]]: full pages are shared, a partly filled last one is copied.  As for GoEnv.copy_slots, destinations are
        pairwise distinct and none is the source of another entry."""
        if _fast is not None:
            rc = _fast.cache_fork(self._calls["fork"], self._h.value, self._shape, src, dst, status)
            if rc == 0: return
            if rc is not None: _check(rc, "pgxcache_fork")
        n, s = self._list(src, "src")
        self._own(dst, torch.int32, (n,), "dst")
        _check(lib().pgxcache_fork(self._h, n, s, _ptr(dst), self._status(status, n)), "pgxcache_fork")

    def free(self, slots=None):
        """The slots' tokens are given up."""
        if _fast is not None:
            rc = _fast.cache_free(self._calls["free"], self._h.value, self._shape, slots)
            if rc == 0: return
            if rc is not None: _check(rc, "pgxcache_free")
        n, p = self._list(slots)
        _check(lib().pgxcache_free(self._h, n, p), "pgxcache_free")

    def compact(self, used=None):
        """Moves pages so that those in use are the first ones; used (int32 [1]) gets their number."""
        if used is not None: self._own(used, torch.int32, (1,), "used")
        _check(lib().pgxcache_compact(self._h, _ptr(used)), "pgxcache_compact")
