"""Host side of the decoding-step calls without a GPU: descriptions that are refused
before anything is allocated or launched, frequencies, workspaces after failures, the
oracle's own pins, and the binding's refusals."""
import ctypes
import math
import os
import subprocess
from fractions import Fraction

import numpy as np
import pytest

from oracle import decode as ref
from paper_2608_05780_gb300.build import CSRC, INCLUDE, nvcc
from test_cache_host import CDraft, FAKE, _cache, _draft  # noqa: F401

EINVAL, EUNSUPPORTED, ECUDA, ENOMEM = -1, -2, -4, -5
I32, I64, F64, P = ctypes.c_int32, ctypes.c_int64, ctypes.c_double, ctypes.c_void_p


class CRope(ctypes.Structure):
    _fields_ = [("rotary_dim", I32), ("interleaved", I32), ("axes", I32), ("section", I32 * 3), ("scale", ctypes.c_float),
                ("reserved", I32), ("turn", ctypes.c_uint64 * 64)]


class CHeads(ctypes.Structure):
    _fields_ = [(n, I32) for n in ("batch", "tokens", "heads", "head_dim", "dtype", "reserved")] + \
               [("in_stride", I64 * 3), ("out_stride", I64 * 3), ("src", P), ("out", P)]


class CPositions(ctypes.Structure):
    _fields_ = [("at", P), ("first", P), ("stride", I64 * 2)]


class CBeams(ctypes.Structure):
    _fields_ = [(n, I32) for n in ("batch", "beams", "vocab", "n_out", "dtype", "pad", "eos", "reserved")] + \
               [("logits_stride", I64 * 2), ("logits", P), ("scores", P), ("finished", P)]


class CState(ctypes.Structure):
    _fields_ = [("src", P), ("out", P), ("row_bytes", I64)]


def _fill(s, over, **f):
    f.update(over)
    for k, v in f.items():
        setattr(s, k, type(getattr(s, k))(*v) if isinstance(v, tuple) else v)
    return s


def _rope(**kw):
    return _fill(CRope(), kw, rotary_dim=128, axes=1, scale=1.0)


def _heads(**kw):
    return _fill(CHeads(), kw, batch=2, tokens=3, heads=28, head_dim=128, in_stride=(10752, 3584, 128), out_stride=(10752, 3584, 128),
                 src=FAKE, out=FAKE + (1 << 20))


def _keys(**kw):
    return _heads(**{**dict(heads=4, in_stride=(1536, 512, 128), out_stride=(1536, 512, 128), src=FAKE + (2 << 20),
                            out=FAKE + (3 << 20)), **kw})


def _pos(**kw):
    return _fill(CPositions(), kw, at=FAKE + (4 << 20), stride=(6, 3))


def _sel(**kw):
    return _fill(CBeams(), kw, batch=2, beams=4, vocab=32000, n_out=8, eos=2, logits_stride=(128000, 32000), logits=FAKE,
                 scores=FAKE + (1 << 20), finished=FAKE + (2 << 20))


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake") / "libfakedecode.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I" + INCLUDE, "-I" + CSRC, "-I" + cuda,
                    *[os.path.join(here, f) for f in ("fake_cuda.cpp", "fake_cache.cpp", "fake_decode.cpp")],
                    *[os.path.join(CSRC, f) for f in ("evisel_capi.cpp", "evisel_cache.cpp", "evisel_decode.cpp")], "-o", out,
                    "-Wl,-z,defs", "-Wl,-Bsymbolic"], check=True)
    lib = ctypes.CDLL(out)
    lib.evisel_last_error.restype = ctypes.c_char_p
    lib.fake_fail.argtypes = [ctypes.c_char_p, ctypes.c_int]
    lib.evisel_free.argtypes = [P]
    lib.evisel_workspace_bytes.argtypes = [P]
    lib.evisel_workspace_bytes.restype = I64
    lib.evisel_rope_init.argtypes = [P, I32, F64, F64, F64, F64, F64, P]
    return lib


def _at(n):
    return P(FAKE + n)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _rotary(lib, ws=None, rope=_rope(), q=_heads(), k=_keys(), pos=_pos()):
    return lib.evisel_rotary(_ref(rope), _ref(q), _ref(k), _ref(pos), 0, None)


def _append(lib, ws, c=_cache(), rope=_rope(), d=None, pos=None, src=_at(8 << 20), counts=_at(9 << 20), lens_out=_at(10 << 20),
            q_out=_at(11 << 20)):
    d = _draft(k_new=FAKE + (5 << 20), v_new=FAKE + (6 << 20)) if d is None else d
    return lib.evisel_cache_append_rotary(_ref(c), _ref(rope), _ref(d), _ref(_pos() if pos is None else pos), src, counts,
                                          lens_out, q_out, None, ws)


def _select(lib, ws, m=_sel(), score=_at(4 << 20), parent=_at(5 << 20), token=_at(6 << 20), ended=_at(7 << 20)):
    return lib.evisel_beam_select(_ref(m), score, parent, token, ended, None, ws)


def _reorder(lib, ws, c=_cache(batch=8), parent=_at(1 << 20), beams=4, states=None, n=None, table=_at(2 << 20), lens=_at(3 << 20)):
    arr = None if states is None else (CState * max(1, len(states)))(*[CState(*s) for s in states])
    return lib.evisel_cache_reorder(_ref(c), parent, beams, arr, len(states or ()) if n is None else n, table, lens, None, ws)


CALLS = dict(rotary=_rotary, append=_append, select=_select, reorder=_reorder)
BAD_ROPE = [(dict(rotary_dim=0), EUNSUPPORTED), (dict(rotary_dim=24), EUNSUPPORTED), (dict(rotary_dim=144), EUNSUPPORTED),
            (dict(interleaved=2), EINVAL), (dict(axes=2), EUNSUPPORTED), (dict(axes=3), EINVAL),
            (dict(axes=3, section=(-1, 33, 32)), EINVAL), (dict(axes=3, section=(1 << 30, 1 << 30, 1 << 30)), EINVAL),
            (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(reserved=1), EINVAL)]
BAD_POS = [(dict(first=FAKE), EINVAL), (dict(at=FAKE + 2), EINVAL), (dict(at=0, first=FAKE + 1), EINVAL), (dict(stride=(-1, 3)), EINVAL), (dict(stride=(1 << 38, 3)), EINVAL), (dict(stride=(0, 1 << 38)), EINVAL),
           (dict(stride=(6, -3)), EINVAL)]


def _refused(lib, rc, code, launches, ws=None):
    assert rc == code, (rc, lib.evisel_last_error())
    assert lib.evisel_last_error() and lib.fake_decode_launches() == launches and (ws is None or ws.value is None)


@pytest.mark.parametrize("call", ["rotary", "append"])
@pytest.mark.parametrize("what,over,code", [("rope", *x) for x in BAD_ROPE] + [("pos", *x) for x in BAD_POS])
def test_bad_ropes_and_positions(fake, call, what, over, code):
    ws, n = P(None), fake.fake_decode_launches()
    kw = {what: (_rope if what == "rope" else _pos)(**over)}
    _refused(fake, CALLS[call](fake, ctypes.byref(ws), **kw), code, n, ws)


Q1, K1 = FAKE, FAKE + (2 << 20)


@pytest.mark.parametrize("call,kw,code", [
    ("rotary", dict(q=None), EINVAL), ("rotary", dict(rope=None), EINVAL), ("rotary", dict(pos=None), EINVAL),
    ("rotary", dict(q=_heads(head_dim=96)), EUNSUPPORTED), ("rotary", dict(q=_heads(dtype=2)), EUNSUPPORTED),
    ("rotary", dict(q=_heads(batch=-1)), EINVAL), ("rotary", dict(q=_heads(reserved=1)), EINVAL),
    ("rotary", dict(q=_heads(tokens=1 << 30)), EUNSUPPORTED), ("rotary", dict(q=_heads(heads=65536)), EUNSUPPORTED),
    ("rotary", dict(q=_heads(src=0)), EINVAL), ("rotary", dict(q=_heads(out=0)), EINVAL), ("rotary", dict(q=_heads(src=FAKE + 8)), EINVAL),
    ("rotary", dict(q=_heads(in_stride=(10752, 3580, 128))), EINVAL), ("rotary", dict(q=_heads(in_stride=(-8, 3584, 128))), EINVAL),
    ("rotary", dict(q=_heads(out_stride=(10752, 0, 128))), EINVAL), ("rotary", dict(q=_heads(out_stride=(10752, 3584, 64))), EINVAL),
    ("rotary", dict(q=_heads(out=FAKE + 256)), EINVAL), ("rotary", dict(q=_heads(out=FAKE, out_stride=(21504, 7168, 128))), EINVAL),
    ("rotary", dict(k=_keys(batch=3)), EINVAL), ("rotary", dict(k=_keys(tokens=4)), EINVAL), ("rotary", dict(k=_keys(dtype=1)), EINVAL),
    ("rotary", dict(k=_keys(head_dim=64)), EINVAL), ("rotary", dict(q=_heads(out=K1)), EINVAL), ("rotary", dict(k=_keys(out=Q1)), EINVAL),
    ("rotary", dict(k=_keys(out=FAKE + (1 << 20))), EINVAL), ("rotary", dict(rope=_rope(rotary_dim=128), q=_heads(head_dim=64)), EUNSUPPORTED),
    ("append", dict(rope=None), EINVAL), ("append", dict(c=None), EINVAL), ("append", dict(lens_out=None), EINVAL),
    ("append", dict(c=_cache(head_dim=64, k_stride=(32768, 8192, 64)), rope=_rope()), EUNSUPPORTED),
    ("append", dict(c=_cache(lens_stride=(4, 1))), EUNSUPPORTED), ("append", dict(c=_cache(page=48)), EUNSUPPORTED),
    ("append", dict(d=_draft(tokens=-1)), EINVAL), ("append", dict(d=_draft(k_new=0)), EINVAL), ("append", dict(d=_draft(hq=0)), EINVAL),
    ("append", dict(d=_draft(q_stride=(10752, 3584, 100))), EINVAL), ("append", dict(d=_draft(q=FAKE + 8)), EINVAL),
    ("append", dict(q_out=None), EINVAL), ("append", dict(q_out=_at(5 << 20)), EINVAL), ("append", dict(q_out=_at(256)), EINVAL),
    ("append", dict(pos=_pos(at=0)), EINVAL), ("append", dict(pos=_pos(at=FAKE + (10 << 20))), EINVAL),
    ("append", dict(src=None, pos=_pos(at=0, first=FAKE + (10 << 20) + 4)), EINVAL), ("append", dict(lens_out=_at(0)), EINVAL),
    ("select", dict(m=None), EINVAL), ("select", dict(m=_sel(dtype=3)), EUNSUPPORTED), ("select", dict(m=_sel(batch=-1)), EINVAL),
    ("select", dict(m=_sel(beams=0)), EUNSUPPORTED), ("select", dict(m=_sel(beams=65)), EUNSUPPORTED), ("select", dict(m=_sel(n_out=0)), EUNSUPPORTED),
    ("select", dict(m=_sel(n_out=65)), EUNSUPPORTED), ("select", dict(m=_sel(vocab=0)), EUNSUPPORTED),
    ("select", dict(m=_sel(vocab=(1 << 24) + 1)), EUNSUPPORTED), ("select", dict(m=_sel(pad=-1)), EINVAL), ("select", dict(m=_sel(pad=32000)), EINVAL),
    ("select", dict(m=_sel(reserved=1)), EINVAL), ("select", dict(m=_sel(batch=20000)), EUNSUPPORTED), ("select", dict(m=_sel(logits=0)), EINVAL),
    ("select", dict(m=_sel(logits=FAKE + 1)), EINVAL), ("select", dict(m=_sel(dtype=2, logits=FAKE + 2)), EINVAL),
    ("select", dict(m=_sel(logits_stride=(-1, 32000))), EINVAL), ("select", dict(score=None), EINVAL), ("select", dict(parent=None), EINVAL),
    ("select", dict(token=_at((6 << 20) + 2)), EINVAL), ("select", dict(score=_at(1 << 20)), EINVAL), ("select", dict(ended=_at(2 << 20)), EINVAL),
    ("select", dict(parent=_at(511996)), EINVAL), ("select", dict(ended=_at(511999)), EINVAL), ("select", dict(token=_at((5 << 20) + 60)), EINVAL),
    ("select", dict(ended=_at((4 << 20) + 63)), EINVAL), ("select", dict(m=_sel(logits_stride=(1 << 38, 32000))), EINVAL),
    ("select", dict(m=_sel(logits_stride=(128000, 1 << 38))), EINVAL), ("select", dict(m=_sel(logits_stride=(1 << 24, 32000))), EINVAL),
    ("reorder", dict(c=None), EINVAL), ("reorder", dict(beams=0), EUNSUPPORTED), ("reorder", dict(beams=65), EUNSUPPORTED),
    ("reorder", dict(beams=3), EINVAL), ("reorder", dict(parent=None), EINVAL), ("reorder", dict(table=None), EINVAL),
    ("reorder", dict(lens=None), EINVAL), ("reorder", dict(lens=_at((3 << 20) + 2)), EINVAL), ("reorder", dict(n=-1), EUNSUPPORTED),
    ("reorder", dict(n=9), EUNSUPPORTED), ("reorder", dict(n=1), EINVAL), ("reorder", dict(c=_cache(batch=8, lens_stride=(4, 1))), EUNSUPPORTED),
    ("reorder", dict(c=_cache(batch=8, table_stride=(200, 50))), EUNSUPPORTED), ("reorder", dict(table=_at(0)), EINVAL),
    ("reorder", dict(lens=_at(1 << 20)), EINVAL), ("reorder", dict(lens=_at(2 << 20)), EINVAL),
    ("reorder", dict(states=[(FAKE + (5 << 20), FAKE + (5 << 20), 64)]), EINVAL), ("reorder", dict(states=[(0, FAKE, 64)]), EINVAL),
    ("reorder", dict(states=[(FAKE + (5 << 20), FAKE + (6 << 20), -1)]), EINVAL),
    ("reorder", dict(states=[(FAKE + (5 << 20), FAKE + (6 << 20), 64), (FAKE + (7 << 20), FAKE + (6 << 20) + 511, 64)]), EINVAL),
    ("reorder", dict(states=[(FAKE + (i << 45), FAKE + (i << 45) + (1 << 44), (1 << 40) - 1) for i in range(1, 5)]), EUNSUPPORTED),
])
def test_bad_calls_are_refused(fake, call, kw, code):
    ws, n = P(None), fake.fake_decode_launches()
    _refused(fake, CALLS[call](fake, ctypes.byref(ws), **kw), code, n, ws)


@pytest.mark.parametrize("call", ["append", "select", "reorder"])
def test_no_workspace_pointer(fake, call):
    n = fake.fake_decode_launches()
    _refused(fake, CALLS[call](fake, None), EINVAL, n)


def test_calls_that_run(fake):
    """The descriptions above without their faults; in place, without keys, without queries; nothing to do."""
    ws, n = P(None), fake.fake_decode_launches()
    at = ctypes.byref(ws)
    own = dict(out=FAKE)
    run = [lambda: _rotary(fake), lambda: _rotary(fake, k=None), lambda: _rotary(fake, q=_heads(**own), k=_keys(out=K1)),
           lambda: _rotary(fake, pos=_pos(at=0)), lambda: _rotary(fake, pos=_pos(at=0, first=FAKE)),
           # rows of one projection, in place: 28 + 4 + 4 heads
           lambda: _rotary(fake, q=_heads(in_stride=(13824, 4608, 128), out_stride=(13824, 4608, 128), **own),
                           k=_keys(in_stride=(13824, 4608, 128), out_stride=(13824, 4608, 128), src=FAKE + 7168, out=FAKE + 7168)),
           lambda: _append(fake, at), lambda: _append(fake, at, src=None, pos=_pos(at=0)), lambda: _append(fake, at, q_out=_at(0)),
           lambda: _append(fake, at, d=_draft(q=0, k_new=FAKE + (5 << 20)), q_out=None, pos=_pos(at=0)),
           lambda: _append(fake, at, d=_draft(tokens=0, q=0, k_new=0, v_new=0), q_out=None),
           lambda: _select(fake, at), lambda: _select(fake, at, m=_sel(scores=0, finished=0, dtype=1), ended=None),
           lambda: _reorder(fake, at), lambda: _reorder(fake, at, states=[(FAKE + (5 << 20), FAKE + (6 << 20), 64), (0, 0, 0)])]
    for i, f in enumerate(run):
        assert f() == 0, (i, fake.evisel_last_error())
        assert fake.fake_decode_launches() == n + i + 1, i
    n = fake.fake_decode_launches()
    for f in (lambda: _rotary(fake, q=_heads(batch=0), k=_keys(batch=0)), lambda: _rotary(fake, q=_heads(tokens=0, src=0, out=0), k=None),
              lambda: _rotary(fake, q=_heads(heads=0), k=None), lambda: _append(fake, at, c=_cache(batch=0, k=0, v=0, table=0, lens=0)),
              lambda: _select(fake, at, m=_sel(batch=0)), lambda: _reorder(fake, at, c=_cache(batch=0, k=0))):
        assert f() == 0 and fake.fake_decode_launches() == n
    fake.evisel_free(ws)


def test_failures_are_reported(fake):
    """A launch, scratch that cannot grow, a capture in which nothing may be allocated: said, and the next call runs."""
    for call in CALLS:
        ws = P(None)
        fake.fake_fail_decode(1)
        assert CALLS[call](fake, ctypes.byref(ws)) == ECUDA and b"launch" in fake.evisel_last_error()
        assert CALLS[call](fake, ctypes.byref(ws)) == 0
        fake.evisel_free(ws)
    ws = P(None)
    assert _select(fake, ctypes.byref(ws)) == 0
    held = fake.evisel_workspace_bytes(ws)
    large = _sel(batch=64, n_out=64, scores=0, finished=0, logits=FAKE + (64 << 20))
    fake.fake_fail(b"cudaMalloc", 0)
    assert _select(fake, ctypes.byref(ws), m=large) == ENOMEM
    fake.fake_capture(1)
    try:
        assert _select(fake, ctypes.byref(ws), m=large) == EINVAL and b"capture" in fake.evisel_last_error()
        assert _select(fake, ctypes.byref(ws)) == 0
        new = P(None)
        for call in ("append", "select", "reorder"):
            assert CALLS[call](fake, ctypes.byref(new)) == EINVAL and new.value is None
        assert _rotary(fake) == 0
    finally:
        fake.fake_capture(0)
    assert _select(fake, ctypes.byref(ws), m=large) == 0 and fake.evisel_workspace_bytes(ws) > held
    fake.evisel_free(ws)


def test_axes_and_blocks(fake):
    """What the launchers get: pairs by axis, blocks of states of any size."""
    for sections in ((16, 24, 24), (0, 64, 0), (0, 0, 64), (64, 0, 0), (1, 0, 63)):
        assert _rotary(fake, rope=_rope(axes=3, section=sections)) == 0
        assert [fake.fake_axis_of_pair(i) for i in range(64)] == [a for a, n in enumerate(sections) for _ in range(n)]
    assert _rotary(fake) == 0 and {fake.fake_axis_of_pair(i) for i in range(64)} == {0}
    ws = P(None)
    sizes = [1, 16384, 16385, 0, 5]
    states = [(FAKE + ((20 + i) << 20), FAKE + ((40 + i) << 20), s) for i, s in enumerate(sizes)]
    assert _reorder(fake, ctypes.byref(ws), states=states) == 0
    assert [fake.fake_reorder_blocks(i) for i in range(6)] == [32, 40, 48, 64, 64, 72]
    fake.evisel_free(ws)


# --- frequencies ------------------------------------------------------------------------

def _turns(lib, r, base=10000.0, factor=1.0, original=0.0, low=1.0, high=4.0, freqs=None):
    rope = CRope()
    f = None if freqs is None else (F64 * len(freqs))(*freqs)
    assert lib.evisel_rope_init(ctypes.byref(rope), r, base, factor, original, low, high, f) == 0, lib.evisel_last_error()
    assert (rope.rotary_dim, rope.interleaved, rope.axes, rope.scale) == (r, 0, 1, 1.0)
    return list(rope.turn)[:r // 2]


PI = Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50)


@pytest.mark.parametrize("kw", [dict(), dict(base=1e6), dict(factor=4.0), dict(factor=8.0, original=8192.0),
                                dict(factor=32.0, original=4096.0, low=1.0, high=32.0, base=5e5)])
@pytest.mark.parametrize("r", [16, 96, 128])
def test_frequencies(fake, r, kw):
    """2^64 f / 2 pi of the formula's f to 53 bits; a position times it, modulo 2^64, is the angle modulo a turn."""
    got = _turns(fake, r, **kw)
    want = ref.frequencies(r, kw.get("base", 1e4), kw.get("factor", 1.0), kw.get("original", 0), kw.get("low", 1.0), kw.get("high", 4.0))
    for t, f in zip(got, want):
        exact = Fraction(f) / (2 * PI)
        assert abs(Fraction(t, 2 ** 64) - exact) <= exact * Fraction(1, 2 ** 51) + Fraction(1, 2 ** 63)
        for p in (1, -1, 1 << 20, -(1 << 31)):
            angle = Fraction((p * t) % 2 ** 64, 2 ** 64)
            off = (angle - p * exact) % 1
            assert min(off, 1 - off) <= abs(p) * Fraction(1, 2 ** 51)


def test_own_frequencies(fake):
    freqs = [0.0, -1.0, 7.5, 1e-9, 2 * math.pi, 100.0, -1e-300, 3.0]
    for t, f in zip(_turns(fake, 16, base=float("nan"), freqs=freqs), freqs):
        off = (Fraction(t, 2 ** 64) - Fraction(f) / (2 * PI)) % 1
        assert min(off, 1 - off) <= Fraction(1, 2 ** 47)


@pytest.mark.parametrize("args,code", [
    ((24, 1e4, 1.0, 0.0, 1.0, 4.0), EUNSUPPORTED), ((144, 1e4, 1.0, 0.0, 1.0, 4.0), EUNSUPPORTED), ((0, 1e4, 1.0, 0.0, 1.0, 4.0), EUNSUPPORTED),
    ((128, 0.0, 1.0, 0.0, 1.0, 4.0), EINVAL), ((128, float("inf"), 1.0, 0.0, 1.0, 4.0), EINVAL), ((128, 1e4, 0.0, 0.0, 1.0, 4.0), EINVAL),
    ((128, 1e4, float("nan"), 0.0, 1.0, 4.0), EINVAL), ((128, 1e4, 1.0, -1.0, 1.0, 4.0), EINVAL), ((128, 1e4, 2.0, 64.0, 4.0, 4.0), EINVAL),
    ((128, 1e4, 2.0, 64.0, float("nan"), 4.0), EINVAL), ((128, 1e-300, 1e-300, 0.0, 1.0, 4.0), EINVAL)])
def test_bad_frequencies(fake, args, code):
    rope = CRope(scale=5.0)
    assert fake.evisel_rope_init(ctypes.byref(rope), *args, None) == code and fake.evisel_last_error()
    assert rope.scale == 5.0
    assert fake.evisel_rope_init(None, 128, 1e4, 1.0, 0.0, 1.0, 4.0, None) == EINVAL
    bad = (F64 * 8)(*[1.0] * 7, float("inf"))
    assert fake.evisel_rope_init(ctypes.byref(rope), 16, 1e4, 1.0, 0.0, 1.0, 4.0, bad) == EINVAL


# --- the oracle's pins --------------------------------------------------------------------

def test_oracle_rotation():
    """By hand at a quarter turn; lengths of pairs stay; products depend on the distance alone; back is back."""
    quarter = [math.pi / 2] * 8
    x = np.arange(16.0).reshape(1, 1, 1, 16)
    y, size = ref.rotate(x, np.array([[1]]), quarter)
    np.testing.assert_allclose(y[0, 0, 0], [-8, -9, -10, -11, -12, -13, -14, -15, 0, 1, 2, 3, 4, 5, 6, 7], atol=1e-12)
    y, _ = ref.rotate(x, np.array([[1]]), quarter, interleaved=True)
    np.testing.assert_allclose(y[0, 0, 0], [-1, 0, -3, 2, -5, 4, -7, 6, -9, 8, -11, 10, -13, 12, -15, 14], atol=1e-12)
    rng, freqs = np.random.default_rng(0), ref.frequencies(16)
    a, b = rng.standard_normal((2, 1, 2, 1, 24))
    for inter in (False, True):
        for t in (0, 7, 1000):
            ra, _ = ref.rotate(a, np.array([[t, t + 5]]), freqs, inter)
            rb, _ = ref.rotate(b, np.array([[t + 3, t]]), freqs, inter)
            dots = (ra * rb).sum(-1)
            if t == 0:
                first = dots
            np.testing.assert_allclose(dots, first, rtol=1e-9)
            back, _ = ref.rotate(ra, np.array([[t, t + 5]]), freqs, inter, transpose=True)
            np.testing.assert_allclose(back, a, rtol=1e-12, atol=1e-12)
    pos = np.array([[[3, 4]], [[50, 60]], [[7, 8]]])
    y, _ = ref.rotate(a, pos, freqs, sections=(8, 0, 0))
    np.testing.assert_allclose(y, ref.rotate(a, pos[0], freqs)[0])
    y, _ = ref.rotate(a, pos, freqs, sections=(0, 3, 5))
    np.testing.assert_allclose(y[..., 3:8], ref.rotate(a, pos[2], freqs)[0][..., 3:8])
    assert size[0, 0, 0, 0] == 8 and size[0, 0, 0, 15] == 22


def test_oracle_scaling():
    """Fast pairs stay, slow ones are divided, in between they are mixed; a factor of 1 changes nothing."""
    plain, mixed = ref.frequencies(128, 1e4), ref.frequencies(128, 1e4, 8.0, 4096.0)
    turns = [4096 * f / (2 * math.pi) for f in plain]
    assert any(t > 4 for t in turns) and any(t < 1 for t in turns)
    for t, f, g in zip(turns, plain, mixed):
        assert g == f if t >= 4 else math.isclose(g, f / 8) if t <= 1 else f / 8 < g < f
    assert ref.frequencies(64, 1e4, 1.0, 100.0) == ref.frequencies(64) and ref.frequencies(64, factor=2.0)[0] == 0.5


def test_oracle_continuations():
    inf, nan = math.inf, math.nan
    got = ref.continuations([[0.0, 0.0, -inf], [1.0, 1.0, 1.0], [nan, 0, 0], [0, 0, inf]], [-1.0, -inf, -1.0, -1.0])
    assert [(k, v) for _, k, v in got] == [(0, 0), (0, 1)] and math.isclose(got[0][0], -1 - math.log(2))
    got = ref.continuations([[0.0, 3.0], [9.0, 9.0]], [-2.0, -0.5], [False, True], pad=1)
    assert [(k, v) for _, k, v in got] == [(1, 1), (0, 1), (0, 0)]
    total = ref.continuations(np.random.default_rng(0).standard_normal((2, 50)), [math.log(0.25), math.log(0.75)])
    assert math.isclose(sum(math.exp(x) for x, _, _ in total), 1.0)


def test_oracle_donors():
    assert ref.donors([0, 1, 2]) == [(0, 0), (1, 1), (2, 2)] and ref.donors([-1, -1]) == [(0, 0), (1, 1)]
    assert ref.donors([2, 2, 2, 0]) == [(2, 2), (2, 1), (2, 3), (0, 0)]
    assert ref.donors([1, 0]) == [(1, 1), (0, 0)] and ref.donors([0, 0, 0]) == [(0, 0), (0, 1), (0, 2)]
    for seed in range(50):
        rng = np.random.default_rng(seed)
        k = int(rng.integers(1, 65))
        out = ref.donors(rng.integers(-1, k, k).tolist())
        assert sorted(d for _, d in out) == list(range(k))


# --- the binding --------------------------------------------------------------------------

def test_binding_refuses():
    """What the Python calls cannot pass on; CPU tensors are refused as such."""
    import torch

    import paper_2608_05780_gb300 as ev
    from paper_2608_05780_gb300.build import build
    build()
    for bad in (dict(head_dim=96), dict(rotary_dim=192), dict(rotary_dim=0), dict(sections=(1, 2)), dict(sections=(64, 1, 0)),
                dict(sections=(-1, 33, 32)), dict(freqs=[1.0]), dict(rotary_dim=1 << 40)):
        with pytest.raises(ValueError):
            ev.Rotary(**{**dict(head_dim=128), **bad})
    for bad in (dict(rotary_dim=24), dict(base=-1.0), dict(factor=0.0), dict(original=64, low_turns=2.0, high_turns=1.0)):
        with pytest.raises(ev.EviselError):
            ev.Rotary(**{**dict(head_dim=128), **bad})
    rope = ev.Rotary(64)
    x = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    for q, k in ((x, None), (x[0, 0], None), (x, x[0]), (x, x.half())):
        with pytest.raises(ValueError):
            ev.evisel_rotary(rope, q, k)
    with pytest.raises(ValueError):
        ev.evisel_beam_select(torch.zeros((1, 2, 30)), None, 2)
