"""ctypes binding of the decoding-step calls (include/evisel_decode.h): argument marshalling only.

What a decoding step needs around the attention over the paged cache: ``Rotary``
describes a position rotation, evisel_rotary applies it to queries and keys,
evisel_cache_append_rotary appends keys rotated on the way, evisel_beam_select
chooses the beams' continuations and evisel_cache_reorder gives the beams that go
on their caches and other states. Conventions and checks are those of ``cache``.
"""
from __future__ import annotations

import ctypes
import struct

from ._binding import Workspace, _check, _maker, load
from .cache import _DRAFT, _NONE, _get, _i32, _new, _plain, _refuse, _stream

_ROPE = struct.Struct("@6ifi64Q")
_HEADS = struct.Struct("@6i6q2P")
_POSITIONS = struct.Struct("@2P2q")
_BEAMS = struct.Struct("@8i2q3P")
_STATE = struct.Struct("@2Pq")
_calls = None


class _Calls:
    def __init__(self):
        import torch
        lib = load()
        vp, i32, f64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_double
        ws = ctypes.POINTER(vp)
        for name, args in (("rope_init", [vp, i32, f64, f64, f64, f64, f64, vp]),
                           ("rotary", [vp, vp, vp, vp, i32, vp]),
                           ("cache_append_rotary", [vp, vp, vp, vp, vp, vp, vp, vp, vp, ws]),
                           ("beam_select", [vp, vp, vp, vp, vp, vp, ws]),
                           ("cache_reorder", [vp, vp, i32, vp, i32, vp, vp, vp, ws])):
            f = getattr(lib, "evisel_" + name)
            f.argtypes, f.restype = args, i32
            setattr(self, name, f)
        base = _get()
        self.empty, self.i32, self.f32, self.masks, self.dtypes = base.empty, base.i32, base.f32, base.masks, base.dtypes
        self.logits = {**base.dtypes, torch.float32: 2}
        self.bool = torch.bool


def _decode():
    global _calls
    if _calls is None:
        _calls = _Calls()
    return _calls


class Rotary:
    """A position rotation of the first ``rotary_dim`` (all by default) of ``head_dim`` dimensions, pair i at the
    frequency base^(-2 i / rotary_dim), or ``freqs[i]`` radians per position.

    Pairs are (x[i], x[i + rotary_dim / 2]), or with ``interleaved`` (x[2 i], x[2 i + 1]). ``sections`` = (t, h, w):
    positions have three axes, which so many pairs each read. For contexts longer than the trained one: ``factor``
    divides every frequency; with ``original`` (the trained length) only those of pairs that turn less than
    ``high_turns`` times over it, wholly below ``low_turns``. ``scale`` multiplies the rotated dimensions."""

    __slots__ = ("head_dim", "rotary_dim", "interleaved", "sections", "scale", "_packed")

    def __init__(self, head_dim, rotary_dim=None, base=10000.0, interleaved=False, sections=None, factor=1.0, original=0,
                 low_turns=1.0, high_turns=4.0, freqs=None, scale=1.0):
        c = _decode()
        r, _, _ = _i32(head_dim if rotary_dim is None else rotary_dim, 0, 0, "rotary_dim")
        if head_dim not in (64, 128) or not 0 < r <= head_dim:
            _refuse("head_dim must be 64 or 128, rotary_dim at most that")
        table = None
        if freqs is not None:
            freqs = [float(f) for f in freqs]
            if len(freqs) != r // 2:
                _refuse(f"freqs must be {r // 2} numbers")
            table = (ctypes.c_double * len(freqs))(*freqs)
        raw = ctypes.create_string_buffer(_ROPE.size)
        rc = c.rope_init(raw, r, float(base), float(factor), float(original), float(low_turns), float(high_turns), table)
        if rc:
            _check(rc)
        turn = _ROPE.unpack(raw.raw)[8:]
        sec = (0, 0, 0)
        if sections is not None:
            sec = tuple(int(s) for s in sections)
            if len(sec) != 3 or min(sec) < 0 or sum(sec) != r // 2:
                _refuse(f"sections must be three numbers that add up to {r // 2}")
        self.head_dim, self.rotary_dim, self.interleaved, self.scale = int(head_dim), r, bool(interleaved), float(scale)
        self.sections = None if sections is None else sec
        self._packed = _ROPE.pack(r, int(self.interleaved), 1 if sections is None else 3, *sec, self.scale, 0, *turn)


def _positions(rope, positions, first, shape, device):
    """The packed positions of [B, T] tokens."""
    if positions is not None:
        if first is not None:
            _refuse("positions or first, not both")
        want = shape if rope.sections is None else (3, *shape)
        ps = positions.stride()
        if not (positions.dtype == _calls.i32 and positions.shape == want and positions.device == device
                and (ps[-1] == 1 or shape[1] <= 1)):
            _refuse(f"positions must be int32 {list(want)} on the device of q and k, tokens contiguous")
        return _POSITIONS.pack(positions.data_ptr(), 0, ps[0] if len(want) == 3 else 0, ps[-2])
    if first is None:
        return _POSITIONS.pack(0, 0, 0, 0)
    if not (first.dtype == _calls.i32 and first.shape == shape[:1] and first.device == device and first.is_contiguous()):
        _refuse("first must be contiguous int32 [B] on the device of q and k")
    return _POSITIONS.pack(0, first.data_ptr(), 0, 0)


def _heads(rope, x, out, shape, batch, tokens, empty, what, c):
    """(the output, made where there is none, the packed heads x [B, T, H, d] or [T, H, d])."""
    s, dtype, d = x.stride(), x.dtype, rope.head_dim
    heads = shape[-2]
    if not (shape[-1] == d and dtype in c.dtypes and x.is_cuda and (s[-1] == 1 or 0 in shape)):
        _refuse(f"{what} must be CUDA [B, T, H, {d}] or [T, H, {d}] of bf16 or fp16, d contiguous")
    if out is None:
        out = empty(shape, dtype=dtype, device=x.device)
        o0, o1, o2 = tokens * heads * d, heads * d, d
    else:
        o = out.stride()
        if out is not x and not (out.shape == shape and out.dtype == dtype and out.device == x.device and (o[-1] == 1 or 0 in shape)):
            _refuse(f"the output of {what} must have its shape, type and device, d contiguous")
        o0, o1, o2 = o[:3] if len(o) == 4 else (0, o[0], o[1])
    s0, s1, s2 = s[:3] if len(s) == 4 else (0, s[0], s[1])
    return out, _HEADS.pack(batch, tokens, heads, d, c.dtypes[dtype], 0, s0, s1, s2, o0, o1, o2, x.data_ptr(), out.data_ptr())


def evisel_rotary(rope, q, k=None, positions=None, first=None, transpose=False, q_out=None, k_out=None, stream=None):
    """Queries q [B, T, hq, d] and keys k [B, T, hkv, d] (or [T, H, d] each, of any strides with d contiguous) rotated
    to their positions: int32 ``positions`` [B, T] (or [T]; with a rope of three sections [3, B, T], [3, T]), or
    ``first`` int32 [B] (or [1]) and on, or 0 and on. ``transpose`` applies the transposed matrix: the gradients of q
    and k from those of the results. The call records none by itself: what it returns does not require one, also where q
    and k do. ``q_out`` and ``k_out`` may be q and k themselves.

    Returns (q_out, k_out), None without k."""
    c = _decode()
    shape, k_shape = q.shape, None if k is None else k.shape
    if len(shape) not in (3, 4) or (k is not None and not (len(k_shape) == len(shape) and k_shape[:-2] == shape[:-2]
                                                           and k.dtype == q.dtype and k.device == q.device)):
        _refuse("q and k must be [B, T, H, d] or [T, H, d], of one batch, tokens, type and device")
    batch, tokens = (1, shape[0]) if len(shape) == 3 else shape[:2]
    if len(shape) == 3 and positions is not None and positions.dim():
        positions = positions.unsqueeze(-2)
    pos = _positions(rope, positions, first, (batch, tokens), q.device)
    empty = _maker(c.empty, stream)
    q_out, packed = _heads(rope, q, q_out, shape, batch, tokens, empty, "q", c)
    k_packed = None
    if k is not None:
        k_out, k_packed = _heads(rope, k, k_out, k_shape, batch, tokens, empty, "k", c)
    elif k_out is not None:
        _refuse("k_out without k")
    rc = c.rotary(rope._packed, packed, k_packed, pos, 1 if transpose else 0, _stream(q, stream))
    if rc:
        _check(rc)
    return q_out, k_out


def evisel_cache_append_rotary(cache, rope, k_new, v_new, q=None, positions=None, first=None, src=None, counts=None,
                               lens_out=None, q_out=None, ws=None, stream=None):
    """evisel_cache_append of keys that are rotated on the way: new token j stands at ``positions`` [B, T] (with a
    rope of three sections [3, B, T]), or the i-th appended one at ``first`` [B] + i, or (neither) at its place in the cache, lens + i. With
    ``q`` [B, T, hq, d] the step's queries are rotated in the same call, all T of each sequence (beside ``src`` only
    with ``positions``).

    Returns (lens int32 [B], q_out [B, T, hq, d] or None, ws)."""
    c = _decode()
    batch = cache.batch
    shape = (batch, k_new.shape[1] if k_new.dim() > 1 else -1, cache.hkv, cache.head_dim)
    if rope.head_dim != cache.head_dim:
        _refuse("the rope's head_dim must be the cache's")
    ks, kp = _new(cache, k_new, shape, "k_new")
    vs, vp = _new(cache, v_new, shape, "v_new")
    pos = _positions(rope, positions, first, shape[:2], cache.device)
    empty = _maker(c.empty, stream)
    qs, hq, qp, qo = _NONE, cache.hkv, 0, 0
    if q is not None:
        qs = q.stride()
        if not (q.dim() == 4 and q.shape[:2] == shape[:2] and q.shape[3] == cache.head_dim and q.dtype == cache.dtype
                and q.device == cache.device and qs[3] == 1):
            _refuse("q must be [B, T, hq, d] of the cache's type and device, d contiguous")
        hq, qp = q.shape[2], q.data_ptr()
        if q_out is None:
            q_out = empty(q.shape, dtype=q.dtype, device=q.device)
            qo = q_out.data_ptr()
        else:
            qo = _plain(cache, q_out, cache.dtype, q.shape, "q_out")
    elif q_out is not None:
        _refuse("q_out without q")
    if lens_out is None:
        lens_out = empty((batch,), dtype=c.i32, device=cache.device)
        out_p = lens_out.data_ptr()
    else:
        out_p = _plain(cache, lens_out, c.i32, (batch,), "lens_out")
    src_p = 0 if src is None else _plain(cache, src, c.i32, shape[:2], "src")
    counts_p = 0 if counts is None else _plain(cache, counts, c.i32, (batch,), "counts")
    draft = _DRAFT.pack(shape[1], hq, 0.0, 0, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], 0, 0,
                        qp, kp, vp, 0, 0)
    ws = Workspace() if ws is None else ws
    rc = c.cache_append_rotary(cache._packed, rope._packed, draft, pos, src_p, counts_p, out_p, qo, _stream(cache, stream),
                               ctypes.byref(ws.ptr))
    if rc:
        _check(rc)
    return lens_out, q_out, ws


def evisel_beam_select(logits, scores=None, n_out=None, finished=None, eos=-1, pad=0, ws=None, stream=None):
    """The ``n_out`` (as many as beams by default) highest continuations of each sequence over its beams and the
    vocabulary, from logits [B, K, V] (bf16, fp16 or fp32, V contiguous) and the beams' summed log-probabilities
    ``scores`` fp32 [B, K] (0 by default): score + log softmax, descending, ties to the lower beam, then the lower
    token. ``finished`` bool [B, K]: beams that have ended go on once, with the token ``pad`` and their score.

    Returns (scores fp32 [B, n], parent int32 [B, n], token int32 [B, n], finished bool [B, n], ws): finished where
    the parent is, where the token is ``eos``, and where there are no more continuations (parent and token -1, score
    -inf)."""
    c = _decode()
    if not (logits.dim() == 3 and logits.is_cuda and logits.dtype in c.logits and (logits.stride()[2] == 1 or logits.shape[2] <= 1)):
        _refuse("logits must be CUDA [B, K, V] of bf16, fp16 or fp32, V contiguous")
    batch, beams, vocab = logits.shape
    n, eos, pad = _i32(beams if n_out is None else n_out, eos, pad, "n_out, eos and pad")
    device, s_p, f_p = logits.device, 0, 0
    if scores is not None:
        if not (scores.dtype == c.f32 and scores.shape == (batch, beams) and scores.device == device and scores.is_contiguous()):
            _refuse("scores must be contiguous fp32 [B, K] on the logits' device")
        s_p = scores.data_ptr()
    if finished is not None:
        if not (finished.dtype in c.masks and finished.shape == (batch, beams) and finished.device == device
                and finished.is_contiguous()):
            _refuse("finished must be contiguous bool or uint8 [B, K] on the logits' device")
        f_p = finished.data_ptr()
    empty, shape = _maker(c.empty, stream), (batch, max(0, n))
    score_out = empty(shape, dtype=c.f32, device=device)
    parent = empty(shape, dtype=c.i32, device=device)
    token = empty(shape, dtype=c.i32, device=device)
    ended = empty(shape, dtype=c.bool, device=device)
    ls = logits.stride()
    packed = _BEAMS.pack(batch, beams, vocab, n, c.logits[logits.dtype], pad, eos, 0, ls[0], ls[1], logits.data_ptr(), s_p, f_p)
    ws = Workspace() if ws is None else ws
    rc = c.beam_select(packed, score_out.data_ptr(), parent.data_ptr(), token.data_ptr(), ended.data_ptr(),
                       _stream(logits, stream), ctypes.byref(ws.ptr))
    if rc:
        _check(rc)
    return score_out, parent, token, ended, ws


def evisel_cache_reorder(cache, parent, states=(), table_out=None, lens_out=None, states_out=None, ws=None, stream=None):
    """The beams that go on: ``parent`` int32 [G, K] names, for each of the cache's G groups of K sequences, the one
    of its group that sequence j takes over from (negative: itself). Full pages are shared, the page in progress is
    copied into a page of a sequence without a child, so that every sequence keeps pages of its own to append to. Full pages
    that only a sequence without a child had are in the cache's table, but not in the new one: free for whoever keeps
    count of pages. Each of ``states`` (contiguous tensors [G K, ...]) is gathered by parent.

    Returns (table int32 [G K, n], lens int32 [G K], states, ws), to be assigned to the cache."""
    c = _decode()
    batch, n = cache.batch, cache.max_tokens // cache.page
    beams = parent.shape[1] if parent.dim() == 2 else -1
    if not (beams > 0 and parent.dtype == c.i32 and parent.shape[0] * beams == batch and parent.device == cache.device
            and parent.is_contiguous()):
        _refuse("parent must be contiguous int32 [G, K] on the cache's device, G K its batch")
    empty = _maker(c.empty, stream)
    outs = [empty(x.shape, dtype=x.dtype, device=x.device) for x in states] if states_out is None else list(states_out)
    if len(outs) != len(states):
        _refuse("states_out must have as many tensors as states")
    packed = b""
    for x, y in zip(states, outs):
        if not (x.dim() > 0 and x.shape[0] == batch and x.device == cache.device and x.is_contiguous()
                and y.shape == x.shape and y.dtype == x.dtype and y.device == x.device and y.is_contiguous()):
            _refuse("states must be contiguous [G K, ...] on the cache's device, their outputs alike")
        packed += _STATE.pack(x.data_ptr(), y.data_ptr(), x.nbytes // batch if batch else 0)
    if table_out is None:
        table_out = empty((batch, n), dtype=c.i32, device=cache.device)
        table_p = table_out.data_ptr()
    else:
        table_p = _plain(cache, table_out, c.i32, (batch, n), "table_out")
    if lens_out is None:
        lens_out = empty((batch,), dtype=c.i32, device=cache.device)
        lens_p = lens_out.data_ptr()
    else:
        lens_p = _plain(cache, lens_out, c.i32, (batch,), "lens_out")
    ws = Workspace() if ws is None else ws
    rc = c.cache_reorder(cache._packed, parent.data_ptr(), beams, packed, len(outs), table_p, lens_p, _stream(cache, stream),
                         ctypes.byref(ws.ptr))
    if rc:
        _check(rc)
    return table_out, lens_out, outs, ws
