"""ctypes binding of the paged-cache calls (include/evisel_cache.h): argument marshalling only.

``Cache`` is the handle of a cache's tensors; the functions carry the C ABI's
names and, like the probe's, take an optional workspace and return it last.
Lengths, tables, tree bits and counts stay on the device: no call waits for it,
and what they hold is checked by the kernels (``evisel_status(ws)`` answers
EVISEL_EBOUNDS, -7, where a length, page id or index was out of range).

``stream`` (a torch.cuda.Stream) takes the place of the current one. What a call
reads must be ready there; the tensors that it returns are made on it.

A decoding step's calls take a few microseconds on the device, so that the
checks here are plain comparisons, their messages formed only when one fails.
"""
from __future__ import annotations

import ctypes
import struct

from ._binding import Workspace, _check, _maker, load

_CACHE = struct.Struct("@8i10q5P")
_DRAFT = struct.Struct("@iifi11q5P")
_NONE = (0, 0, 0, 0)
_calls = None           # the library's functions, torch's names and lookups: filled by the first call


class _Calls:
    def __init__(self):
        import torch
        lib = load()
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
        ws = ctypes.POINTER(vp)
        for name, args in (("attention", [vp, vp, vp, vp, vp, ws]),
                           ("evidence", [vp, vp, vp, vp, vp, i64, i32, vp, ws]),
                           ("evict", [vp, vp, i64, vp, i32, i32, i32, vp, vp, i64, vp, ws]),
                           ("append", [vp, vp, vp, vp, vp, vp, ws]),
                           ("select", [vp, vp, i32, i32, i32, vp, vp, vp, vp, ws])):
            f = getattr(lib, "evisel_cache_" + name)
            f.argtypes, f.restype = args, i32
            setattr(self, name, f)
        self.empty, self.zeros, self.i32, self.f32 = torch.empty, torch.zeros, torch.int32, torch.float32
        self.dtypes = {torch.bfloat16: 0, torch.float16: 1}
        self.masks = (torch.bool, torch.uint8)
        self.current_device = torch.cuda.current_device
        self.raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)


def _get():
    global _calls
    if _calls is None:
        _calls = _Calls()
    return _calls


def _refuse(what):
    raise ValueError(what)


def _i32(a, b, c, what):
    """Three whole numbers for the C ABI, which refuses negative ones (ctypes would wrap those past 32 bits)."""
    a, b, c = int(a), int(b), int(c)
    if not -1 <= (a | b | c) >> 31 <= 0:
        _refuse(f"{what} must fit 32 bits")
    return a, b, c


class Cache:
    """A paged cache: ``k`` and ``v`` pages [P, hkv, page, d] (bf16 or fp16, any strides with d contiguous: pages
    stored [P, page, hkv, d] are passed transposed), ``table`` int32 [B, n] or [B, hkv, n] of page ids, ``lens`` int32
    [B] or [B, hkv] of cached tokens, and optionally ``k_mean`` [P, hkv, d] of the pages' mean keys.

    The handle holds the tensors; assign one (``lens``, ``table``, ``k``, ``v``, ``k_mean``) to replace it.
    """

    __slots__ = ("_k", "_v", "_k_mean", "device", "dtype", "batch", "hkv", "page", "head_dim", "max_tokens", "_pool",
                 "_table", "_lens", "_chosen", "_packed")

    def __init__(self, k, v, table, lens, k_mean=None):
        c = _get()
        if not (k.dim() == 4 and k.shape == v.shape):
            _refuse("k and v must be pages [P, hkv, page, d] of one shape")
        if not (k.is_cuda and k.dtype in c.dtypes and v.dtype == k.dtype and v.device == k.device):
            _refuse("k and v must be CUDA tensors of bf16 or fp16 on one device")
        ks, vs = k.stride(), v.stride()
        if not (ks[3] == 1 and vs[3] == 1):
            _refuse("d must be contiguous in k and v")
        pages, hkv, page, d = k.shape
        if k_mean is not None and not (k_mean.shape == (pages, hkv, d) and k_mean.dtype == k.dtype
                                       and k_mean.device == k.device and k_mean.is_contiguous()):
            _refuse("k_mean must be contiguous [P, hkv, d], of k's type and device")
        self._k, self._v, self._k_mean, self.device, self.dtype = k, v, k_mean, k.device, k.dtype
        self.hkv, self.page, self.head_dim = hkv, page, d
        self._pool = (pages, c.dtypes[k.dtype], ks[:3], vs[:3], k.data_ptr(), v.data_ptr(),
                      0 if k_mean is None else k_mean.data_ptr())
        self._set(table, lens)

    def _set(self, table, lens):
        i32 = _calls.i32
        ts, ls, batch, hkv = table.stride(), lens.stride(), lens.shape[0] if lens.dim() else -1, self.hkv
        if not (lens.dtype == i32 and lens.device == self.device and (lens.shape == (batch,) or lens.shape == (batch, hkv))):
            _refuse("lens must be int32 [B] or [B, hkv] on the cache's device")
        n = table.shape[-1] if table.dim() else -1
        if not (table.dtype == i32 and table.device == self.device and (table.shape == (batch, n) or table.shape == (batch, hkv, n))):
            _refuse("table must be int32 [B, n] or [B, hkv, n] on the cache's device")
        if not (ts[-1] == 1 or n <= 1):
            _refuse("table rows must be contiguous")
        pages, dtype, ks, vs, kp, vp, mp = self._pool
        self._table, self._lens, self._chosen, self.batch, self.max_tokens = table, lens, None, batch, n * self.page
        self._packed = _CACHE.pack(batch, hkv, self.head_dim, self.page, pages, n, dtype, 0, *ks, *vs,
                                   ts[0], ts[1] if len(ts) == 3 else 0, ls[0], ls[1] if len(ls) == 2 else 0,
                                   kp, vp, table.data_ptr(), lens.data_ptr(), mp)

    def _tensors(self):
        if self._table is None:                  # a choice's: cut out of its buffer when somebody asks
            rows, n = self.batch * self.hkv, self.max_tokens // self.page
            self._table = self._chosen[:rows * n].view(self.batch, self.hkv, n)
            self._lens = self._chosen[rows * n:].view(self.batch, self.hkv)
        return self._table, self._lens

    @property
    def table(self):
        return self._tensors()[0]

    @table.setter
    def table(self, table):
        self._set(table, self.lens)

    @property
    def lens(self):
        return self._tensors()[1]

    @lens.setter
    def lens(self, lens):
        self._set(self.table, lens)

    def _replace_pages(self, k, v, k_mean):
        new = Cache(k, v, *self._tensors(), k_mean)          # with its checks; this one stays as it was where they fail
        for name in Cache.__slots__:
            setattr(self, name, getattr(new, name))

    @property
    def k(self):
        return self._k

    @k.setter
    def k(self, k):
        self._replace_pages(k, self._v, self._k_mean)

    @property
    def v(self):
        return self._v

    @v.setter
    def v(self, v):
        self._replace_pages(self._k, v, self._k_mean)

    @property
    def k_mean(self):
        return self._k_mean

    @k_mean.setter
    def k_mean(self, k_mean):
        self._replace_pages(self._k, self._v, k_mean)

    def _same_pages(self):
        c = object.__new__(Cache)
        c._k, c._v, c._k_mean, c.device, c.dtype = self._k, self._v, self._k_mean, self.device, self.dtype
        c.hkv, c.page, c.head_dim, c._pool = self.hkv, self.page, self.head_dim, self._pool
        return c

    def view(self, table, lens):
        """The same pages under another table and lengths."""
        c = self._same_pages()
        c._set(table, lens)
        return c

    def _choice(self, n, empty):
        """A view of n pages per (sequence, head), its table and lengths to be written; the addresses of both."""
        c, batch, hkv = self._same_pages(), self.batch, self.hkv
        c._table = c._lens = None
        c._chosen = empty((batch * hkv * (n + 1),), dtype=_calls.i32, device=self.device)
        c.batch, c.max_tokens = batch, n * self.page
        table_p = c._chosen.data_ptr()
        lens_p = table_p + 4 * batch * hkv * n
        pages, dtype, ks, vs, kp, vp, mp = self._pool
        c._packed = _CACHE.pack(batch, hkv, self.head_dim, self.page, pages, n, dtype, 0, *ks, *vs, hkv * n, n, hkv, 1,
                                kp, vp, table_p, lens_p, mp)
        return c, table_p, lens_p


def _new(cache, x, shape, what):
    """Strides and address of new keys or values."""
    s = x.stride()
    if not (x.shape == shape and x.dtype == cache.dtype and x.device == cache.device and s[3] == 1):
        _refuse(f"{what} must be [B, T, hkv, d] = {list(shape)} of the cache's type and device, d contiguous")
    return s, x.data_ptr()


def _plain(cache, x, dtype, shape, what):
    """Address of a contiguous tensor of this type and shape."""
    if not (x.dtype == dtype and x.shape == shape and x.device == cache.device and x.is_contiguous()):
        _refuse(f"{what} must be contiguous {dtype} {list(shape)} on the cache's device")
    return x.data_ptr()


def _draft(cache, q, k_new, v_new, tree, drafted, scale):
    qs, sh = q.stride(), q.shape
    if not (len(sh) == 4 and sh[0] == cache.batch and sh[3] == cache.head_dim and q.dtype == cache.dtype
            and q.device == cache.device and qs[3] == 1):
        _refuse("q must be [B, T, hq, d] of the cache's type and device, d contiguous")
    batch, tokens, hq, d = sh
    ks = vs = _NONE
    kp = vp = tp = dp = t0 = t1 = 0
    if k_new is not None or v_new is not None:
        if k_new is None or v_new is None:
            _refuse("k_new and v_new go together")
        shape = (batch, tokens, cache.hkv, d)
        ks, kp = _new(cache, k_new, shape, "k_new")
        vs, vp = _new(cache, v_new, shape, "v_new")
    if tree is not None:
        words, ts = (tokens + 31) // 32, tree.stride()
        if tree.shape == (batch, tokens, words):
            t0, t1 = ts[0], ts[1]
        elif tree.shape == (tokens, words):
            t1 = ts[0]
        else:
            _refuse(f"tree must be int32 bit words [B, {tokens}, {words}] or [{tokens}, {words}]")
        if not (tree.dtype == _calls.i32 and tree.device == cache.device and (ts[-1] == 1 or words <= 1)):
            _refuse("tree must be int32 with contiguous rows on the cache's device")
        tp = tree.data_ptr()
    if drafted is not None:
        dp = _plain(cache, drafted, _calls.i32, (batch,), "drafted")
    return _DRAFT.pack(tokens, hq, scale, 0, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], t0, t1,
                       q.data_ptr(), kp, vp, tp, dp)


def _stream(cache, stream):
    index = cache.device.index
    if index != _calls.current_device():
        _refuse("the cache's device must be the current one")
    return _calls.raw_stream(index) if stream is None else stream.cuda_stream


def evisel_cache_attention(cache, q, k_new=None, v_new=None, tree=None, drafted=None, ws=None, o=None, lse=None,
                           softmax_scale=0.0, stream=None):
    """Attention of T drafted tokens q [B, T, hq, d] of each sequence over its cache and over those of the drafted
    k_new, v_new [B, T, hkv, d] that ``tree`` allows: int32 bit words [B, T, ceil(T / 32)] (or one tree [T, ...] for
    all), bit j of row t set where token t attends drafted token j; None: a chain (j <= t). ``drafted`` int32 [B]:
    tokens that a sequence has drafted, T each by default. The strides of q, k_new and v_new are free but for d's.

    Returns (o [B, T, hq, d], lse [hq, B, T] fp32, ws)."""
    draft = _draft(cache, q, k_new, v_new, tree, drafted, softmax_scale)
    batch, tokens, hq, d = q.shape
    empty = _maker(_calls.empty, stream)
    o_p = (empty((batch, tokens, hq, d), dtype=cache.dtype, device=cache.device) if o is None else o)
    lse_p = (empty((hq, batch, tokens), dtype=_calls.f32, device=cache.device) if lse is None else lse)
    if o is not None:
        _plain(cache, o, cache.dtype, q.shape, "o")
    if lse is not None:
        _plain(cache, lse, _calls.f32, (hq, batch, tokens), "lse")
    ws = Workspace() if ws is None else ws
    rc = _calls.attention(cache._packed, draft, o_p.data_ptr(), lse_p.data_ptr(), _stream(cache, stream), ctypes.byref(ws.ptr))
    if rc:
        _check(rc)
    return o_p, lse_p, ws


def evisel_cache_evidence(cache, q, lse, acc=None, use=None, drafted=None, accumulate=False, ws=None,
                          softmax_scale=0.0, stream=None):
    """Attention weight of the queries q [B, T, hq, d] per cached token, summed over the rows and the heads of each
    KV group, from the row normalisers ``lse`` [hq, B, T] of evisel_cache_attention. ``use`` bool [B, T]: the rows
    that count. ``acc`` fp32 [B, hkv, n] (zeros up to cache.max_tokens by default) is overwritten, or with
    ``accumulate`` added to, up to each sequence's length.

    Returns (acc, ws)."""
    draft = _draft(cache, q, None, None, None, drafted, softmax_scale)
    batch, tokens, hq, _ = q.shape
    lse_p = _plain(cache, lse, _calls.f32, (hq, batch, tokens), "lse")
    if acc is None:
        acc = _maker(_calls.zeros, stream)((batch, cache.hkv, cache.max_tokens), dtype=_calls.f32, device=cache.device)
    n = acc.shape[-1] if acc.dim() else 0
    acc_p = _plain(cache, acc, _calls.f32, (batch, cache.hkv, n), "acc")
    use_p = 0
    if use is not None:
        if use.dtype not in _calls.masks:
            _refuse("use must be bool or uint8")
        use_p = _plain(cache, use, use.dtype, (batch, tokens), "use")
    ws = Workspace() if ws is None else ws
    rc = _calls.evidence(cache._packed, draft, lse_p, use_p, acc_p, n, 1 if accumulate else 0, _stream(cache, stream),
                         ctypes.byref(ws.ptr))
    if rc:
        _check(rc)
    return acc, ws


def evisel_cache_evict(cache, acc, out, budget, sink=0, recent=0, kept=None, acc_out=None, ws=None, stream=None):
    """Cuts every (sequence, KV head) of ``cache`` down to ``budget`` tokens, into the first slots of the cache
    ``out`` (other pages): the first ``sink``, the last ``recent`` and those with the largest ``acc`` [B, hkv, n].
    out.lens, and out.k_mean where there is one, are written.

    Returns (kept int32 [B, hkv, budget] with -1 past the tokens kept, acc_out [B, hkv, out.max_tokens], ws)."""
    batch, hkv = cache.batch, cache.hkv
    budget, sink, recent = _i32(budget, sink, recent, "budget, sink and recent")
    n = acc.shape[-1] if acc.dim() else 0
    acc_p = _plain(cache, acc, _calls.f32, (batch, hkv, n), "acc")
    if not (out.device == cache.device and out.batch == batch and out.hkv == hkv):
        _refuse("out must have the cache's batch, heads and device")
    shape = (batch, hkv, budget if budget > 0 else 0)
    empty = _maker(_calls.empty, stream)
    if kept is None:
        kept = empty(shape, dtype=_calls.i32, device=cache.device)
        kept_p = kept.data_ptr()
    else:
        kept_p = _plain(cache, kept, _calls.i32, shape, "kept")
    if acc_out is None:
        m = out.max_tokens
        acc_out = empty((batch, hkv, m), dtype=_calls.f32, device=cache.device)
        acc_out_p = acc_out.data_ptr()
    else:
        m = acc_out.shape[-1] if acc_out.dim() else 0
        acc_out_p = _plain(cache, acc_out, _calls.f32, (batch, hkv, m), "acc_out")
    ws = Workspace() if ws is None else ws
    rc = _calls.evict(cache._packed, acc_p, n, out._packed, budget, sink, recent, kept_p, acc_out_p, m,
                      _stream(cache, stream), ctypes.byref(ws.ptr))
    if rc:
        _check(rc)
    return kept, acc_out, ws


def evisel_cache_append(cache, k_new, v_new, src=None, counts=None, lens_out=None, ws=None, stream=None):
    """Appends the first ``counts`` (int32 [B], T by default) of the tokens k_new, v_new [B, T, hkv, d], or of those
    that ``src`` (int32 [B, T]) names, to each sequence, and forms the means of the touched pages again.
    cache.lens is not written: the new lengths are returned, to be assigned to it.

    Returns (lens int32 [B], ws)."""
    batch = cache.batch
    shape = (batch, k_new.shape[1] if k_new.dim() > 1 else -1, cache.hkv, cache.head_dim)
    ks, kp = _new(cache, k_new, shape, "k_new")
    vs, vp = _new(cache, v_new, shape, "v_new")
    if lens_out is None:
        lens_out = _maker(_calls.empty, stream)((batch,), dtype=_calls.i32, device=cache.device)
        out_p = lens_out.data_ptr()
    else:
        out_p = _plain(cache, lens_out, _calls.i32, (batch,), "lens_out")
    src_p = 0 if src is None else _plain(cache, src, _calls.i32, shape[:2], "src")
    counts_p = 0 if counts is None else _plain(cache, counts, _calls.i32, (batch,), "counts")
    draft = _DRAFT.pack(shape[1], cache.hkv, 0.0, 0, 0, 0, 0, ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], 0, 0,
                        0, kp, vp, 0, 0)
    ws = Workspace() if ws is None else ws
    rc = _calls.append(cache._packed, draft, src_p, counts_p, out_p, _stream(cache, stream), ctypes.byref(ws.ptr))
    if rc:
        _check(rc)
    return lens_out, ws


def evisel_cache_select(cache, q, n_select, sink=0, recent=1, drafted=None, ws=None, stream=None):
    """Chooses ``n_select`` pages for every (sequence, KV head): the first ``sink``, the last ``recent`` and those
    whose mean key (cache.k_mean) has the largest product with a query of q [B, T, hq, d].

    Returns (view, pages, ws): a Cache of the chosen pages for evisel_cache_attention, and their logical numbers
    int32 [B, hkv, n_select], ascending, -1 past them."""
    draft = _draft(cache, q, None, None, None, drafted, 0.0)
    n_select, sink, recent = _i32(n_select, sink, recent, "n_select, sink and recent")
    n = max(0, n_select)
    empty = _maker(_calls.empty, stream)
    pages = empty((cache.batch, cache.hkv, n), dtype=_calls.i32, device=cache.device)
    view, table_p, lens_p = cache._choice(n, empty)
    ws = Workspace() if ws is None else ws
    rc = _calls.select(cache._packed, draft, n_select, sink, recent, pages.data_ptr(), table_p, lens_p,
                       _stream(cache, stream), ctypes.byref(ws.ptr))
    if rc:
        _check(rc)
    return view, pages, ws
