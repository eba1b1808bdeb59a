"""ctypes binding of the paged-cache calls (include/evisel_cache.h): argument marshalling only.

``Cache`` is the handle of a cache's tensors; the functions carry the C ABI's
names and, like the probe's, take an optional workspace and return it last.
Lengths, tables, tree bits and counts stay on the device: no call waits for it,
and what they hold is checked by the kernels (``evisel_status(ws)`` answers
EVISEL_EBOUNDS, -7, where a length, page id or index was out of range).
"""
from __future__ import annotations

import ctypes
import struct

from ._binding import Workspace, _check, _stream_handle, load

_CACHE = struct.Struct("@8i10q5P")
_DRAFT = struct.Struct("@iifi11q5P")
_declared = False
_DTYPES = {}


def _lib():
    global _declared
    lib = load()
    if not _declared:
        import torch
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
        ws = ctypes.POINTER(vp)
        for name, args in (("attention", [vp, vp, vp, vp, vp, ws]),
                           ("evidence", [vp, vp, vp, vp, vp, i64, i32, vp, ws]),
                           ("evict", [vp, vp, i64, vp, i32, i32, i32, vp, vp, i64, vp, ws]),
                           ("append", [vp, vp, vp, vp, vp, vp, ws]),
                           ("select", [vp, vp, i32, i32, i32, vp, vp, vp, vp, ws])):
            f = getattr(lib, "evisel_cache_" + name)
            f.argtypes, f.restype = args, i32
        _DTYPES.update({torch.bfloat16: 0, torch.float16: 1})
        _declared = True
    return lib


def _need(ok, what):
    if not ok:
        raise ValueError(what)


class Cache:
    """A paged cache: ``k`` and ``v`` pages [P, hkv, page, d] (bf16 or fp16, any strides with d contiguous: pages
    stored [P, page, hkv, d] are passed transposed), ``table`` int32 [B, n] or [B, hkv, n] of page ids, ``lens`` int32
    [B] or [B, hkv] of cached tokens, and optionally ``k_mean`` [P, hkv, d] of the pages' mean keys.

    The handle holds the tensors; assign ``lens`` or ``table`` to replace one.
    """

    __slots__ = ("k", "v", "k_mean", "device", "shape", "_table", "_lens", "_packed")

    def __init__(self, k, v, table, lens, k_mean=None):
        import torch
        _lib()
        _need(k.dim() == 4 and k.shape == v.shape, "k and v must be pages [P, hkv, page, d] of one shape")
        _need(k.is_cuda and k.dtype in _DTYPES and v.dtype == k.dtype and v.device == k.device,
              "k and v must be CUDA tensors of bf16 or fp16 on one device")
        _need(k.stride(3) == 1 and v.stride(3) == 1, "d must be contiguous in k and v")
        if k_mean is not None:
            _need(k_mean.shape == (k.shape[0], k.shape[1], k.shape[3]) and k_mean.dtype == k.dtype
                  and k_mean.device == k.device and k_mean.is_contiguous(),
                  "k_mean must be contiguous [P, hkv, d], of k's type and device")
        self.k, self.v, self.k_mean, self.device = k, v, k_mean, k.device
        self.shape = tuple(k.shape)
        self._set(table, lens, torch.int32)

    def _set(self, table, lens, i32):
        n_pages, hkv, page, d = self.shape
        for x, dim, what in ((table, 2, "table"), (lens, 1, "lens")):
            _need(x.dtype == i32 and x.device == self.device and x.dim() in (dim, dim + 1)
                  and x.shape[0] == lens.shape[0] and (x.dim() == dim or x.shape[1] == hkv),
                  f"{what} must be int32 [B{', n' * (dim - 1)}] or [B, hkv{', n' * (dim - 1)}] on the cache's device")
        _need(table.stride(-1) == 1 or table.shape[-1] <= 1, "table rows must be contiguous")
        k, v, km = self.k, self.v, self.k_mean
        self._table, self._lens = table, lens
        self._packed = _CACHE.pack(
            lens.shape[0], hkv, d, page, n_pages, table.shape[-1], _DTYPES[k.dtype], 0, *k.stride()[:3],
            *v.stride()[:3], table.stride(0), table.stride(1) if table.dim() == 3 else 0, lens.stride(0),
            lens.stride(1) if lens.dim() == 2 else 0, k.data_ptr(), v.data_ptr(), table.data_ptr(), lens.data_ptr(),
            0 if km is None else km.data_ptr())

    @property
    def table(self):
        return self._table

    @table.setter
    def table(self, table):
        self._set(table, self._lens, self._lens.dtype)

    @property
    def lens(self):
        return self._lens

    @lens.setter
    def lens(self, lens):
        self._set(self._table, lens, self._table.dtype)

    @property
    def batch(self):
        return self._lens.shape[0]

    @property
    def hkv(self):
        return self.shape[1]

    @property
    def max_tokens(self):
        """Tokens that a table row can hold."""
        return self._table.shape[-1] * self.shape[2]

    def view(self, table, lens):
        """The same pages under another table and lengths."""
        c = object.__new__(Cache)
        c.k, c.v, c.k_mean, c.device, c.shape = self.k, self.v, self.k_mean, self.device, self.shape
        c._set(table, lens, self._lens.dtype)
        return c


def _check_new(cache, x, tokens, what):
    _need(x.dim() == 4 and x.shape[0] == cache.batch and x.shape[2:] == (cache.shape[1], cache.shape[3])
          and (tokens is None or x.shape[1] == tokens), f"{what} must be [B, T, hkv, d]")
    _need(x.dtype == cache.k.dtype and x.device == cache.device and x.stride(3) == 1,
          f"{what} must have the cache's type and device, d contiguous")


def _i32(cache, x, shape, what):
    import torch
    _need(x.dtype == torch.int32 and x.shape == shape and x.device == cache.device and x.is_contiguous(),
          f"{what} must be contiguous int32 {list(shape)} on the cache's device")
    return x.data_ptr()


def _f32(cache, x, shape, what):
    import torch
    _need(x.dtype == torch.float32 and x.shape == shape and x.device == cache.device and x.is_contiguous(),
          f"{what} must be contiguous float32 {list(shape)} on the cache's device")
    return x.data_ptr()


def _draft(cache, q, k_new, v_new, tree, drafted, scale):
    import torch
    _need(q.dim() == 4 and q.shape[0] == cache.batch and q.shape[3] == cache.shape[3] and q.dtype == cache.k.dtype
          and q.device == cache.device and q.stride(3) == 1,
          "q must be [B, T, hq, d] of the cache's type and device, d contiguous")
    tokens, hq = q.shape[1], q.shape[2]
    qs = q.stride()
    ks = vs = (0, 0, 0)
    kp = vp = tp = dp = t0 = t1 = 0
    _need((k_new is None) == (v_new is None), "k_new and v_new go together")
    if k_new is not None:
        _check_new(cache, k_new, tokens, "k_new")
        _check_new(cache, v_new, tokens, "v_new")
        ks, vs, kp, vp = k_new.stride(), v_new.stride(), k_new.data_ptr(), v_new.data_ptr()
    if tree is not None:
        words = -(-tokens // 32)
        _need(tree.dtype == torch.int32 and tree.device == cache.device and tree.dim() in (2, 3)
              and tree.shape[-2:] == (tokens, words) and (tree.dim() == 2 or tree.shape[0] == cache.batch)
              and (tree.stride(-1) == 1 or words <= 1),
              f"tree must be int32 bit words [B, {tokens}, {words}] or [{tokens}, {words}] on the cache's device")
        tp, t1, t0 = tree.data_ptr(), tree.stride(-2), tree.stride(0) if tree.dim() == 3 else 0
    if drafted is not None:
        dp = _i32(cache, drafted, (cache.batch,), "drafted")
    return _DRAFT.pack(tokens, hq, scale, 0, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], t0, t1,
                       q.data_ptr(), kp, vp, tp, dp)


def _call(cache, name, ws, stream, *args):
    import torch
    lib = _lib()
    _need(cache.device.index == torch.cuda.current_device(), "the cache's device must be the current one")
    ws = Workspace() if ws is None else ws
    _check(getattr(lib, name)(*args, _stream_handle(stream), ctypes.byref(ws.ptr)))
    return ws


def evisel_cache_attention(cache, q, k_new=None, v_new=None, tree=None, drafted=None, ws=None, o=None, lse=None,
                           softmax_scale=0.0, stream=None):
    """Attention of T drafted tokens q [B, T, hq, d] of each sequence over its cache and over those of the drafted
    k_new, v_new [B, T, hkv, d] that ``tree`` allows: int32 bit words [B, T, ceil(T / 32)] (or one tree [T, ...] for
    all), bit j of row t set where token t attends drafted token j; None: a chain (j <= t). ``drafted`` int32 [B]:
    tokens that a sequence has drafted, T each by default. The strides of q, k_new and v_new are free but for d's.

    Returns (o [B, T, hq, d], lse [hq, B, T] fp32, ws)."""
    import torch
    draft = _draft(cache, q, k_new, v_new, tree, drafted, softmax_scale)
    batch, tokens, hq, d = q.shape
    if o is None:
        o = torch.empty((batch, tokens, hq, d), dtype=q.dtype, device=q.device)
    else:
        _need(o.shape == q.shape and o.dtype == q.dtype and o.device == q.device and o.is_contiguous(),
              "o must be contiguous [B, T, hq, d] of q's type")
    if lse is None:
        lse = torch.empty((hq, batch, tokens), dtype=torch.float32, device=q.device)
    else:
        _f32(cache, lse, (hq, batch, tokens), "lse")
    ws = _call(cache, "evisel_cache_attention", ws, stream, cache._packed, draft, o.data_ptr(), lse.data_ptr())
    return o, lse, ws


def evisel_cache_evidence(cache, q, lse, acc=None, use=None, drafted=None, accumulate=False, ws=None,
                          softmax_scale=0.0, stream=None):
    """Attention weight of the queries q [B, T, hq, d] per cached token, summed over the rows and the heads of each
    KV group, from the row normalisers ``lse`` [hq, B, T] of evisel_cache_attention. ``use`` bool [B, T]: the rows
    that count. ``acc`` fp32 [B, hkv, n] (cache.max_tokens by default) is overwritten, or with ``accumulate`` added
    to, up to each sequence's length.

    Returns (acc, ws)."""
    import torch
    draft = _draft(cache, q, None, None, None, drafted, softmax_scale)
    batch, tokens, hq, _ = q.shape
    lse_p = _f32(cache, lse, (hq, batch, tokens), "lse")
    if acc is None:
        acc = torch.zeros((batch, cache.hkv, cache.max_tokens), dtype=torch.float32, device=q.device)
    _need(acc.dim() == 3, "acc must be [B, hkv, n]")
    acc_p = _f32(cache, acc, (batch, cache.hkv, acc.shape[2]), "acc")
    use_p = 0
    if use is not None:
        _need(use.dtype in (torch.bool, torch.uint8) and use.shape == (batch, tokens) and use.device == cache.device
              and use.is_contiguous(), "use must be contiguous bool [B, T] on the cache's device")
        use_p = use.data_ptr()
    ws = _call(cache, "evisel_cache_evidence", ws, stream, cache._packed, draft, lse_p, use_p, acc_p, acc.shape[2],
               int(bool(accumulate)))
    return acc, ws


def evisel_cache_evict(cache, acc, out, budget, sink=0, recent=0, kept=None, acc_out=None, ws=None, stream=None):
    """Cuts every (sequence, KV head) of ``cache`` down to ``budget`` tokens, into the first slots of the cache
    ``out`` (other pages): the first ``sink``, the last ``recent`` and those with the largest ``acc`` [B, hkv, n].
    out.lens, and out.k_mean where there is one, are written.

    Returns (kept int32 [B, hkv, budget] with -1 past the tokens kept, acc_out [B, hkv, out.max_tokens], ws)."""
    import torch
    _need(acc.dim() == 3, "acc must be [B, hkv, n]")
    acc_p = _f32(cache, acc, (cache.batch, cache.hkv, acc.shape[2]), "acc")
    _need(out.device == cache.device, "out must be on the cache's device")
    _need(out.batch == cache.batch and out.hkv == cache.hkv, "out must have the cache's batch and heads")
    if kept is None:
        kept = torch.empty((cache.batch, cache.hkv, max(0, int(budget))), dtype=torch.int32, device=cache.device)
    if acc_out is None:
        acc_out = torch.empty((cache.batch, cache.hkv, out.max_tokens), dtype=torch.float32, device=cache.device)
    _need(acc_out.dim() == 3, "acc_out must be [B, hkv, n]")
    ws = _call(cache, "evisel_cache_evict", ws, stream, cache._packed, acc_p, acc.shape[2], out._packed, int(budget),
               int(sink), int(recent), _i32(cache, kept, (cache.batch, cache.hkv, max(0, int(budget))), "kept"),
               _f32(cache, acc_out, (cache.batch, cache.hkv, acc_out.shape[2]), "acc_out"), acc_out.shape[2])
    return kept, acc_out, ws


def evisel_cache_append(cache, k_new, v_new, src=None, counts=None, lens_out=None, ws=None, stream=None):
    """Appends the first ``counts`` (int32 [B], T by default) of the tokens k_new, v_new [B, T, hkv, d], or of those
    that ``src`` (int32 [B, T]) names, to each sequence, and forms the means of the touched pages again.
    cache.lens is not written: the new lengths are returned, to be assigned to it.

    Returns (lens int32 [B], ws)."""
    import torch
    _check_new(cache, k_new, None, "k_new")
    tokens = k_new.shape[1]
    _check_new(cache, v_new, tokens, "v_new")
    if lens_out is None:
        lens_out = torch.empty((cache.batch,), dtype=torch.int32, device=cache.device)
    ks, vs = k_new.stride(), v_new.stride()
    draft = _DRAFT.pack(tokens, cache.hkv, 0.0, 0, 0, 0, 0, ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], 0, 0,
                        0, k_new.data_ptr(), v_new.data_ptr(), 0, 0)
    ws = _call(cache, "evisel_cache_append", ws, stream, cache._packed, draft,
               0 if src is None else _i32(cache, src, (cache.batch, tokens), "src"),
               0 if counts is None else _i32(cache, counts, (cache.batch,), "counts"),
               _i32(cache, lens_out, (cache.batch,), "lens_out"))
    return lens_out, ws


def evisel_cache_select(cache, q, n_select, sink=0, recent=1, drafted=None, ws=None, stream=None):
    """Chooses ``n_select`` pages for every (sequence, KV head): the first ``sink``, the last ``recent`` and those
    whose mean key (cache.k_mean) has the largest product with a query of q [B, T, hq, d].

    Returns (view, pages, ws): a Cache of the chosen pages for evisel_cache_attention, and their logical numbers
    int32 [B, hkv, n_select], ascending, -1 past them."""
    import torch
    draft = _draft(cache, q, None, None, None, drafted, 0.0)
    batch, hkv = cache.batch, cache.hkv
    out = torch.empty((2, batch, hkv, max(0, int(n_select))), dtype=torch.int32, device=cache.device)
    lens = torch.empty((batch, hkv), dtype=torch.int32, device=cache.device)
    pages, table = out[0], out[1]
    ws = _call(cache, "evisel_cache_select", ws, stream, cache._packed, draft, int(n_select), int(sink), int(recent),
               pages.data_ptr(), table.data_ptr(), lens.data_ptr())
    return cache.view(table, lens), pages, ws
