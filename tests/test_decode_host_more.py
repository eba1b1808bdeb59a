"""Host side of the decoding-step calls, continued: outputs over what a call reads, pages that leave the tables."""
import ctypes
import itertools
import math
import os
import subprocess
from fractions import Fraction

import numpy as np
import pytest

from oracle import decode as ref
from paper_2608_05780_gb300.build import CSRC, INCLUDE, nvcc
from test_cache_host import FAKE, _append as _plain_append, _cache, _draft
from test_decode_host import _append, _at, _heads, _keys, _pos, _rope, _rotary, _turns, PI, fake  # noqa: F401

EINVAL = -1
MB = 1 << 20


def _run(fake, f):
    """The call's return code; nothing was launched where it was refused."""
    ws, n = ctypes.c_void_p(None), (fake.fake_launches(), fake.fake_decode_launches())
    rc = f(ctypes.byref(ws))
    assert (rc == 0) != ((fake.fake_launches(), fake.fake_decode_launches()) == n), fake.evisel_last_error()
    fake.evisel_free(ws)
    return rc


# --- ranges ---------------------------------------------------------------------------

def _bytes(p, size, width, sizes, strides):
    out = set()
    for at in itertools.product(*map(range, sizes)):
        first = p + size * sum(a * s for a, s in zip(at, strides))
        out.update(range(first, first + size * width))
    return out


def test_ranges(tmp_path):
    """Against all bytes one by one: nested dimensions in any order, repeated ones, of one place and of none; dimensions
    that step into one another count as one piece at least where they meet."""
    out = str(tmp_path / "libranges.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I" + INCLUDE, "-I" + CSRC, "-I" + cuda,
                    os.path.join(here, "fake_ranges.cpp"), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    U64, I64 = ctypes.c_uint64, ctypes.c_int64
    lib.ranges_meet.argtypes = [U64, U64, U64, ctypes.c_int, I64, ctypes.c_int, ctypes.POINTER(I64), ctypes.POINTER(I64)]
    rng, met = np.random.default_rng(0), 0
    for _ in range(4000):
        n, size, width, p = int(rng.integers(0, 4)), int(rng.choice([1, 2, 4])), int(rng.integers(1, 5)), int(rng.integers(40, 60))
        sizes, strides, step = rng.integers(1, 4, n).tolist(), [], width
        nested = rng.random() < 0.8
        for s in sizes:
            step += int(rng.integers(0, 4))
            strides.append(step if nested else int(rng.integers(0, 9)))
            step += (s - 1) * step
            if nested and rng.random() < 0.2:
                strides[-1] = 0
        if n and rng.random() < 0.1:
            sizes[int(rng.integers(n))] = 0
        order = rng.permutation(n)
        sizes, strides = [sizes[i] for i in order], [strides[i] for i in order]
        all_ = _bytes(p, size, width, sizes, strides)
        for _ in range(12):
            begin = int(rng.integers(30, max(all_, default=60) + 10))
            end = begin + int(rng.integers(0, 12))
            want = any(begin <= x < end for x in all_)
            got = lib.ranges_meet(begin, end, p, size, width, n, (I64 * 3)(*sizes), (I64 * 3)(*strides))
            assert bool(got) == want if nested else bool(got) >= want, (begin, end, p, size, width, sizes, strides)
            met += want
    assert met > 1000
    far = (I64 * 3)(1 << 50, 1 << 62, 1 << 40)               # strides that no memory has
    assert lib.ranges_meet(40, 50, 40, 4, 1, 3, (I64 * 3)(7, 7, 7), far) == 1
    assert lib.ranges_meet(50, 60, 40, 4, 1, 3, (I64 * 3)(7, 7, 7), far) == 0
    assert lib.ranges_meet(0, 60, 0, 4, 1, 1, (I64 * 3)(7), (I64 * 3)(1)) == 0          # no tensor


# --- outputs over what a call reads ------------------------------------------------------

LENS, TABLE = FAKE + 30 * MB, FAKE + 40 * MB


@pytest.mark.parametrize("call", [_plain_append, _append])
@pytest.mark.parametrize("stride,batch,at,code", [
    (1, 2, 1, EINVAL), (1, 2, -1, EINVAL), (1, 2, 0, EINVAL), (1, 2, 2, 0), (1, 2, -2, 0), (5, 2, 1, 0), (5, 2, 4, EINVAL), (5, 2, 5, EINVAL),
    (5, 2, 6, 0), (0, 2, 1, 0), (0, 2, -1, EINVAL), (0, 1, 1, 0)])
def test_lengths_over_lengths(fake, call, stride, batch, at, code):  # noqa: F811
    """An append writes lens_out while its other blocks still read the cache's lengths."""
    kw = dict(c=_cache(lens=LENS, table=TABLE, lens_stride=(stride, 0), batch=batch), d=_draft(k_new=FAKE + 5 * MB, v_new=FAKE + 6 * MB),
              lens_out=ctypes.c_void_p(LENS + 4 * at), src=_at(8 * MB), counts=_at(9 * MB))
    assert _run(fake, lambda ws: call(fake, ws, **kw)) == code


@pytest.mark.parametrize("stride,at,code", [
    (50, 49, EINVAL), (50, 99, EINVAL), (50, -1, EINVAL), (50, 100, 0), (50, -2, 0), (60, 52, 0), (60, 59, EINVAL), (0, 50, 0), (0, 49, EINVAL)])
def test_lengths_over_the_table(fake, stride, at, code):  # noqa: F811
    """And the table, of 50 pages to a sequence."""
    c = _cache(lens=LENS, table=TABLE, table_stride=(stride, 0))
    assert _run(fake, lambda ws: _append(fake, ws, c=c, lens_out=ctypes.c_void_p(TABLE + 4 * at))) == code


SRC, COUNTS, LENS_OUT, AT, K, V, MEAN, Q_OUT = (FAKE + i * MB for i in (41, 42, 43, 44, 50, 60, 70, 80))
Q_BYTES = 2 * 3 * 28 * 128 * 2      # of two sequences, three tokens, 28 heads of 128


@pytest.mark.parametrize("over,at,code", [
    (dict(), Q_OUT, 0), (dict(), LENS + 4, EINVAL), (dict(), LENS - Q_BYTES, 0), (dict(), LENS - Q_BYTES + 16, EINVAL), (dict(), LENS + 16, 0),
    (dict(), TABLE + 384, EINVAL), (dict(), TABLE + 400, 0), (dict(), SRC, EINVAL), (dict(), SRC + 32, 0), (dict(), COUNTS, EINVAL),
    (dict(), COUNTS + 16, 0), (dict(), LENS_OUT - 16, EINVAL), (dict(), LENS_OUT + 16, 0), (dict(), AT - Q_BYTES + 16, EINVAL),
    (dict(pos=dict(at=AT, stride=(0, 65536))), AT + 16, 0), (dict(pos=dict(at=AT, stride=(0, 65536))), AT + 4 * 65536 - 16, EINVAL),
    (dict(pos=dict(at=AT, stride=(65536, 3)), axes=3), AT + 8 * 65536, EINVAL), (dict(pos=dict(at=AT, stride=(65536, 3)), axes=3), AT + 4 * 65536 + 32, 0),
    (dict(pos=dict(at=AT, stride=(65536, 3))), AT + 8 * 65536, 0), (dict(pos=dict(at=0, first=AT), src=0), AT, EINVAL),
    (dict(pos=dict(at=0, first=AT), src=0), AT + 16, 0),
    (dict(), K, EINVAL), (dict(), K + 100 * 65536, 0), (dict(), K + 100 * 65536 - 16, EINVAL), (dict(), V + 99 * 65536, EINVAL), (dict(), MEAN + 102384, EINVAL),
    (dict(), MEAN + 102400, 0), (dict(mean=0), MEAN, 0),
    (dict(k_stride=(131072, 8192, 128)), K + 65536, 0), (dict(k_stride=(131072, 8192, 128)), K + 262144 - 16, EINVAL),   # every second page of 64 KB
    (dict(k_stride=(131072, 256, 1024)), K + 131072, 0), (dict(k_stride=(131072, 256, 1024)), K + 131072 - 512, EINVAL)])
def test_queries_over_what_an_append_reads(fake, over, at, code):  # noqa: F811
    """Rotated queries are written while other blocks read lengths, tables and positions and write pages; gaps between them
    are nobody's."""
    over = dict(over)
    pos = _pos(**{**dict(at=AT, stride=(0, 3)), **over.pop("pos", {})})
    rope = _rope(axes=3, section=(16, 24, 24)) if over.pop("axes", 1) == 3 else _rope()
    src = ctypes.c_void_p(over.pop("src", SRC))
    c = _cache(**{**dict(lens=LENS, table=TABLE, k=K, v=V, k_mean=over.pop("mean", MEAN)), **over})
    kw = dict(c=c, rope=rope, pos=pos, src=src, counts=ctypes.c_void_p(COUNTS), lens_out=ctypes.c_void_p(LENS_OUT),
              q_out=ctypes.c_void_p(at))
    assert _run(fake, lambda ws: _append(fake, ws, **kw)) == code


ROW = 2 * (28 * 128 + 8)            # of a sequence: 28 heads of 128, and 16 bytes that hold its position


@pytest.mark.parametrize("pos,axes,heads,code", [
    (dict(at=AT, stride=(6, 3)), 1, {}, 0), (dict(at=Q_OUT, stride=(6, 3)), 1, {}, EINVAL), (dict(at=Q_OUT + Q_BYTES - 4, stride=(6, 3)), 1, {}, EINVAL),
    (dict(at=Q_OUT + Q_BYTES, stride=(6, 3)), 1, {}, 0), (dict(at=Q_OUT - 24, stride=(6, 3)), 1, {}, 0), (dict(at=Q_OUT - 20, stride=(6, 3)), 1, {}, EINVAL),
    (dict(at=Q_OUT - 4096, stride=(1024, 3)), 3, {}, EINVAL), (dict(at=Q_OUT - 4096, stride=(20000, 3)), 3, {}, 0),
    (dict(at=0, first=Q_OUT + 4), 1, {}, EINVAL), (dict(at=0, first=Q_OUT - 8), 1, {}, 0), (dict(at=0, first=Q_OUT - 4), 1, {}, EINVAL),
    (dict(at=Q_OUT, stride=(6, 3)), 1, dict(heads=0), 0),
    # one token of each of 200 sequences, whose rows hold queries and position
    (dict(at=Q_OUT + ROW - 16, stride=(0, ROW // 4)), 1, dict(batch=200, tokens=1, out_stride=(ROW // 2, 0, 128)), 0),
    (dict(at=Q_OUT + ROW - 20, stride=(0, ROW // 4)), 1, dict(batch=200, tokens=1, out_stride=(ROW // 2, 0, 128)), EINVAL)])
def test_rotated_heads_over_positions(fake, pos, axes, heads, code):  # noqa: F811
    """Of queries, then of keys."""
    rope, pos = _rope(axes=3, section=(16, 24, 24)) if axes == 3 else _rope(), _pos(**pos)
    mine = _heads(**{**dict(out=Q_OUT), **heads})
    far = _heads(**{n: x for n, x in heads.items() if n != "heads"}, out=FAKE + (1 << 44))
    assert _rotary(fake, None, rope, mine, None, pos) == code
    assert _rotary(fake, None, rope, far, None, pos) == 0 and _rotary(fake, None, rope, far, mine, pos) == code
    # Too many sequences to look at one by one, with strides that no memory has.
    many, wide = _heads(out=Q_OUT, batch=1 << 28, tokens=4, out_stride=(1 << 30, 4096, 128)), _pos(at=Q_OUT - 4096, stride=(0, (1 << 38) - 1))
    assert _rotary(fake, None, _rope(), many, None, wide) == EINVAL


def test_rotated_heads_in_the_rows_of_one_tensor(fake):  # noqa: F811
    """Outputs that share rows, and an output beside its input there, share no memory; where they do they are refused."""
    rows = (3 * 4608, 4608, 128)            # two sequences, three tokens, 36 heads
    at = lambda head: Q_OUT + 256 * head    # noqa: E731
    q = lambda head, **kw: _heads(**{**dict(out=at(head), out_stride=rows), **kw})  # noqa: E731
    k = lambda head, **kw: _keys(**{**dict(out=at(head), out_stride=rows), **kw})  # noqa: E731
    run = lambda *a: _rotary(fake, None, _rope(), *a, _pos(at=AT))  # noqa: E731
    assert run(q(0), k(28)) == run(q(0), k(32)) == run(q(8), k(0)) == run(q(8), k(4)) == 0
    assert run(q(0), k(27)) == run(q(8), k(5)) == run(q(0), k(33)) == run(q(0), k(0)) == EINVAL
    assert run(q(0), k(36)) == EINVAL       # the second token's row
    inside = dict(in_stride=rows)
    assert run(q(0), k(28, src=at(32), **inside)) == run(q(0, src=FAKE), k(28, src=at(28), **inside)) == 0
    assert run(q(0), k(28, src=at(30), **inside)) == run(q(0), k(28, src=at(20), **inside)) == EINVAL
    wide = dict(in_stride=(3 * 9216, 9216, 128), out_stride=(3 * 9216, 9216, 128))
    assert run(q(28, src=at(0), **wide), None) == 0 and run(q(27, src=at(0), **wide), None) == EINVAL
    # Heads outside the tokens: 36 x 3 rows of a sequence.
    inner = (3 * 4608, 128, 384)
    assert run(q(0, out_stride=inner), k(3 * 28, out_stride=inner)) == 0
    assert run(q(0, out_stride=inner), k(3 * 28 - 1, out_stride=inner)) == EINVAL
    assert run(q(0), k(3 * 28, out_stride=inner)) == EINVAL         # rows of other strides
    assert run(q(0, out_stride=(10752, 3584, 128)), k(28)) == EINVAL


# --- turns -----------------------------------------------------------------------------

def test_turns_are_as_near_as_documented(fake):  # noqa: F811
    """f / 2 pi: 2 pi in fp64 is off by 0.35 x 2^-53 relative, the quotient by 2^-53 of itself, a negative one's fraction by
    2^-54, the cut by 2^-64; whole turns are dropped exactly. Together below max(1, |f| / 2 pi) 2^-52."""
    rng = np.random.default_rng(0)
    freqs = [0.0, 1.0, -1.0, 2 * math.pi, 7.5, 100.0, -100.0, 1e4, 12345.678, -1e9, 1e-9, -1e-300, 3e-18, 1e15]
    freqs += (rng.standard_normal(498) * 10.0 ** rng.uniform(-6, 8, 498)).tolist()
    for i in range(0, len(freqs), 64):
        part = freqs[i:i + 64]
        for t, f in zip(_turns(fake, 2 * len(part), base=float("nan"), freqs=part), part):
            exact = Fraction(f) / (2 * PI)
            bound = max(Fraction(1), abs(exact)) / 2 ** 52
            for p in (1, -1, 70001, (1 << 31) - 1, -(1 << 31)):
                off = (Fraction((p * t) % 2 ** 64, 2 ** 64) - p * exact) % 1
                assert min(off, 1 - off) <= abs(p) * bound, (f, p)


# --- the oracle's pins -------------------------------------------------------------------

def test_oracle_pages_that_leave():
    """Two beams of 36 tokens that share a page of 16: the second's full page of its own is in no table afterwards, the
    pages in progress stay."""
    cache = dict(k=np.zeros((5, 1, 16, 8)), v=np.zeros((5, 1, 16, 8)), k_mean=None, lens=np.array([36, 36]),
                 table=np.array([[0, 1, 2], [0, 3, 4]]))
    table, lens, _ = ref.reorder(cache, np.array([[0, 0]]))
    assert table.tolist() == [[0, 1, 2], [0, 1, 4]] and lens.tolist() == [36, 36]
    cache.update(table=np.array([[0, 1], [2, 3]]), lens=np.array([20, 20]))
    assert ref.reorder(cache, np.array([[0, 0]]))[0].tolist() == [[0, 1], [0, 3]]
