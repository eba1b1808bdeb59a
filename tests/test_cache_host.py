"""Host side of the paged-cache calls without a GPU: descriptions that are refused
before anything is allocated or launched, the workspace after failures, the
rule that shares units of work over CTAs, and the oracle's own pins."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import cache as ref_cache
from paper_2608_05780_gb300.build import CSRC, INCLUDE, nvcc

EINVAL, EUNSUPPORTED, ECUDA, ENOMEM = -1, -2, -4, -5
FAKE = 0x7F0000000000   # never dereferenced: the launchers are stand-ins
I64x2, I64x3 = ctypes.c_int64 * 2, ctypes.c_int64 * 3


class CCache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "hkv", "head_dim", "page", "n_pages", "max_pages", "dtype",
                                              "reserved")] + \
               [("k_stride", I64x3), ("v_stride", I64x3), ("table_stride", I64x2), ("lens_stride", I64x2)] + \
               [(n, ctypes.c_void_p) for n in ("k", "v", "table", "lens", "k_mean")]


class CDraft(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int32), ("hq", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("reserved", ctypes.c_int32), ("q_stride", I64x3), ("k_new_stride", I64x3), ("v_new_stride", I64x3),
                ("tree_stride", I64x2)] + \
               [(n, ctypes.c_void_p) for n in ("q", "k_new", "v_new", "tree", "drafted")]


def _cache(**kw):
    f = dict(batch=2, hkv=4, head_dim=128, page=64, n_pages=100, max_pages=50, dtype=0, k_stride=(32768, 8192, 128),
             v_stride=(32768, 8192, 128), table_stride=(50, 0), lens_stride=(1, 0), k=FAKE, v=FAKE, table=FAKE, lens=FAKE,
             k_mean=FAKE)
    f.update(kw)
    c = CCache()
    for k, v in f.items():
        setattr(c, k, type(getattr(c, k))(*v) if isinstance(v, tuple) else v)
    return c


def _draft(**kw):
    f = dict(tokens=3, hq=28, softmax_scale=0.0, q_stride=(10752, 3584, 128), k_new_stride=(1536, 512, 128),
             v_new_stride=(1536, 512, 128), tree_stride=(3, 1), q=FAKE, k_new=FAKE, v_new=FAKE, tree=FAKE, drafted=FAKE)
    f.update(kw)
    d = CDraft()
    for k, v in f.items():
        setattr(d, k, type(getattr(d, k))(*v) if isinstance(v, tuple) else v)
    return d


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake") / "libfakecache.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I" + INCLUDE, "-I" + CSRC, "-I" + cuda,
                    os.path.join(here, "fake_cuda.cpp"), os.path.join(here, "fake_cache.cpp"),
                    os.path.join(CSRC, "evisel_capi.cpp"), os.path.join(CSRC, "evisel_cache.cpp"), "-o", out,
                    "-Wl,-z,defs", "-Wl,-Bsymbolic"], check=True)
    lib = ctypes.CDLL(out)
    lib.evisel_last_error.restype = ctypes.c_char_p
    lib.fake_fail.argtypes = [ctypes.c_char_p, ctypes.c_int]
    lib.evisel_free.argtypes = [ctypes.c_void_p]
    lib.evisel_workspace_bytes.argtypes = [ctypes.c_void_p]
    lib.evisel_workspace_bytes.restype = ctypes.c_int64
    return lib


P = ctypes.c_void_p(FAKE)
Q = ctypes.c_void_p(FAKE + 4096)
L64 = ctypes.c_int64


def _attention(lib, ws, c=None, d=None, o=P, lse=P):
    return lib.evisel_cache_attention(ctypes.byref(c or _cache()), ctypes.byref(d or _draft()), o, lse, None, ws)


def _evidence(lib, ws, c=None, d=None, lse=P, acc=P, n=3200):
    return lib.evisel_cache_evidence(ctypes.byref(c or _cache()), ctypes.byref(d or _draft()), lse, None, acc, L64(n), 0, None, ws)


def _evict(lib, ws, c=None, out=None, budget=64, sink=4, recent=8, n=3200, m=64, acc=P, acc_out=Q):
    out = out or _cache(k=FAKE + 8192, lens=FAKE + 64, table=FAKE + 128, page=32, max_pages=2, k_stride=(16384, 4096, 128),
                        v_stride=(16384, 4096, 128))
    return lib.evisel_cache_evict(ctypes.byref(c or _cache()), acc, L64(n), ctypes.byref(out), budget, sink, recent, P,
                                  acc_out, L64(m), None, ws)


def _append(lib, ws, c=None, d=None, src=P, counts=P, lens_out=Q):
    return lib.evisel_cache_append(ctypes.byref(c or _cache()), ctypes.byref(d or _draft()), src, counts, lens_out, None, ws)


def _select(lib, ws, c=None, d=None, n=8, sink=1, recent=2, pages=P):
    return lib.evisel_cache_select(ctypes.byref(c or _cache()), ctypes.byref(d or _draft()), n, sink, recent, pages, P, P, None, ws)


CALLS = dict(attention=_attention, evidence=_evidence, evict=_evict, append=_append, select=_select)

BAD_CACHE = [
    (dict(head_dim=96), EUNSUPPORTED), (dict(page=48), EUNSUPPORTED), (dict(page=256), EUNSUPPORTED),
    (dict(dtype=2), EUNSUPPORTED), (dict(dtype=-1), EUNSUPPORTED), (dict(batch=-1), EINVAL), (dict(hkv=0), EINVAL),
    (dict(n_pages=0), EINVAL), (dict(max_pages=-1), EINVAL), (dict(reserved=1), EINVAL), (dict(k=0), EINVAL),
    (dict(v=0), EINVAL), (dict(table=0), EINVAL), (dict(lens=0), EINVAL), (dict(k=FAKE + 8), EINVAL),
    (dict(k_mean=FAKE + 2), EINVAL), (dict(lens=FAKE + 2), EINVAL), (dict(k_stride=(32768, 8192, 100)), EINVAL),
    (dict(v_stride=(32768, 8192, 0)), EINVAL), (dict(k_stride=(32768, -8192, 128)), EINVAL),
    (dict(k_stride=(1 << 38, 8192, 128)), EINVAL), (dict(table_stride=(-1, 0)), EINVAL), (dict(lens_stride=(1, -1)), EINVAL),
    (dict(batch=70000), EUNSUPPORTED), (dict(batch=20000, hkv=4), EUNSUPPORTED), (dict(max_pages=1 << 25), EUNSUPPORTED),
]
BAD_DRAFT = [
    (dict(tokens=-1), EINVAL), (dict(tokens=1025), EUNSUPPORTED), (dict(hq=27), EUNSUPPORTED), (dict(hq=0), EUNSUPPORTED),
    (dict(hq=4 * 129), EUNSUPPORTED), (dict(softmax_scale=-1.0), EINVAL), (dict(softmax_scale=float("inf")), EINVAL),
    (dict(softmax_scale=float("nan")), EINVAL), (dict(reserved=7), EINVAL), (dict(q=0), EINVAL), (dict(q=FAKE + 8), EINVAL),
    (dict(q_stride=(10752, 3584, 100)), EINVAL), (dict(q_stride=(10752, -8, 128)), EINVAL), (dict(drafted=FAKE + 1), EINVAL),
]


def _refused(lib, rc, code, launches, ws):
    assert rc == code, (rc, lib.evisel_last_error())
    assert lib.evisel_last_error() and lib.fake_launches() == launches and ws.value is None


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("over,code", BAD_CACHE)
def test_bad_caches_are_refused(fake, call, over, code):
    ws, n = ctypes.c_void_p(None), fake.fake_launches()
    _refused(fake, CALLS[call](fake, ctypes.byref(ws), c=_cache(**over)), code, n, ws)


@pytest.mark.parametrize("call", ["attention", "evidence", "select"])
@pytest.mark.parametrize("over,code", BAD_DRAFT)
def test_bad_drafts_are_refused(fake, call, over, code):
    ws, n = ctypes.c_void_p(None), fake.fake_launches()
    _refused(fake, CALLS[call](fake, ctypes.byref(ws), d=_draft(**over)), code, n, ws)


@pytest.mark.parametrize("call,kw,code", [
    ("attention", dict(o=None), EINVAL), ("attention", dict(lse=None), EINVAL), ("attention", dict(o=ctypes.c_void_p(FAKE + 4)), EINVAL),
    ("attention", dict(d=_draft(v_new=0)), EINVAL), ("attention", dict(d=_draft(k_new=FAKE + 4)), EINVAL),
    ("attention", dict(d=_draft(k_new_stride=(1536, 512, 4))), EINVAL), ("attention", dict(d=_draft(tree=FAKE + 2)), EINVAL),
    ("attention", dict(d=_draft(tree_stride=(-1, 1))), EINVAL),
    ("attention", dict(c=_cache(batch=16000, max_pages=1 << 23)), EUNSUPPORTED),
    ("evidence", dict(acc=None), EINVAL), ("evidence", dict(lse=None), EINVAL), ("evidence", dict(n=-1), EINVAL),
    ("evict", dict(budget=0), EINVAL), ("evict", dict(sink=-1), EINVAL), ("evict", dict(sink=40, recent=25), EINVAL),
    ("evict", dict(budget=65, m=65), EINVAL), ("evict", dict(m=63), EINVAL), ("evict", dict(acc=None), EINVAL),
    ("evict", dict(acc_out=P), EINVAL), ("evict", dict(out=_cache(batch=3)), EINVAL), ("evict", dict(out=_cache(hkv=2)), EINVAL),
    ("evict", dict(out=_cache(dtype=1)), EINVAL), ("evict", dict(out=_cache()), EINVAL),
    ("evict", dict(c=_cache(lens_stride=(4, 1))), EINVAL),
    ("append", dict(lens_out=None), EINVAL), ("append", dict(lens_out=P), EINVAL), ("append", dict(src=ctypes.c_void_p(FAKE + 1)), EINVAL),
    ("append", dict(d=_draft(k_new=0)), EINVAL), ("append", dict(d=_draft(tokens=-1)), EINVAL),
    ("append", dict(c=_cache(lens_stride=(4, 1))), EUNSUPPORTED), ("append", dict(c=_cache(table_stride=(200, 50))), EUNSUPPORTED),
    ("select", dict(recent=0), EINVAL), ("select", dict(n=2), EINVAL), ("select", dict(sink=-1), EINVAL),
    ("select", dict(pages=None), EINVAL), ("select", dict(c=_cache(k_mean=0)), EINVAL),
    ("select", dict(c=_cache(max_pages=8193)), EUNSUPPORTED),
])
def test_bad_calls_are_refused(fake, call, kw, code):
    ws, n = ctypes.c_void_p(None), fake.fake_launches()
    _refused(fake, CALLS[call](fake, ctypes.byref(ws), **kw), code, n, ws)


@pytest.mark.parametrize("call", CALLS)
def test_null_descriptions(fake, call):
    ws = ctypes.c_void_p(None)
    f = getattr(fake, "evisel_cache_" + call)
    d, c = ctypes.byref(_draft()), ctypes.byref(_cache())
    tail = dict(attention=(P, P, None), evidence=(P, None, P, L64(9), 0, None), append=(P, P, Q, None),
                select=(8, 1, 2, P, P, P, None))
    if call == "evict":
        assert f(None, P, L64(9), c, 8, 0, 0, P, Q, L64(8), None, ctypes.byref(ws)) == EINVAL
        assert f(c, P, L64(9), None, 8, 0, 0, P, Q, L64(8), None, ctypes.byref(ws)) == EINVAL
        assert _evict(fake, None) == EINVAL
    else:
        assert f(None, d, *tail[call], ctypes.byref(ws)) == EINVAL
        assert f(c, None, *tail[call], ctypes.byref(ws)) == EINVAL
        assert CALLS[call](fake, None) == EINVAL
    assert ws.value is None


@pytest.mark.parametrize("call", CALLS)
def test_nothing_to_do(fake, call):
    """An empty batch, and (where that means nothing) no drafted token: no launch, no workspace."""
    n, ws = fake.fake_launches(), ctypes.c_void_p(None)
    kw = dict(c=_cache(batch=0, k=0, v=0, table=0, lens=0))
    if call == "evict":
        kw["out"] = _cache(batch=0, k=0)
    assert CALLS[call](fake, ctypes.byref(ws), **kw) == 0 and fake.fake_launches() == n and ws.value is None
    if call == "attention":
        assert _attention(fake, ctypes.byref(ws), d=_draft(tokens=0, q=0)) == 0 and fake.fake_launches() == n


@pytest.mark.parametrize("name", [b"cudaMalloc", b"encode"])
def test_a_failed_attention_leaves_a_workspace_that_works(fake, name):
    """Scratch that cannot grow, a map that cannot be made: the call says so, and the next one runs."""
    ws = ctypes.c_void_p(None)
    assert _attention(fake, ctypes.byref(ws)) == 0
    held = fake.evisel_workspace_bytes(ws)
    assert held > 0
    large = dict(c=_cache(batch=64), d=_draft(tokens=200, q_stride=(1 << 20, 3584, 128)))
    n = fake.fake_launches()
    fake.fake_fail(name, 0)
    assert _attention(fake, ctypes.byref(ws), **large) == (ENOMEM if name == b"cudaMalloc" else ECUDA)
    assert fake.fake_launches() == n
    assert _attention(fake, ctypes.byref(ws)) == 0 and _attention(fake, ctypes.byref(ws), **large) == 0
    assert fake.evisel_workspace_bytes(ws) > held
    fake.evisel_free(ws)


@pytest.mark.parametrize("call", CALLS)
def test_a_failed_launch_is_reported(fake, call):
    ws = ctypes.c_void_p(None)
    fake.fake_fail_launch(1)
    assert CALLS[call](fake, ctypes.byref(ws)) == ECUDA and b"launch" in fake.evisel_last_error()
    assert CALLS[call](fake, ctypes.byref(ws)) == 0
    fake.evisel_free(ws)


# --- the split of ragged work ----------------------------------------------------

def _ctas(total, n_ctas, least, problems):
    if problems * 8 <= n_ctas:
        return max(1, min(n_ctas // problems, -(-total // (least * problems)))) * problems
    return max(1, min(n_ctas, -(-total // least)))


def _begin(i, total, ctas):
    q, r = divmod(total, ctas)
    return i * q + i * r // ctas


@pytest.mark.parametrize("seed", range(60))
def test_split_covers_every_key_once(seed):
    """The rule of the kernels (cache_common.cuh), in Python: every key tile of every problem falls to one CTA, the
    CTAs that the join looks for are those that have some, and no two parts share a partial."""
    rng = np.random.default_rng(seed)
    problems, lead, least, n_ctas = int(rng.integers(1, 400)), int(rng.integers(0, 3)), int(rng.integers(1, 4)), 304
    tiles = rng.integers(0, rng.choice([2, 5, 70, 1100]), problems)
    units = np.where(tiles > 0, tiles + lead, 0)
    first = np.concatenate([[0], np.cumsum(units)])
    total = int(first[-1])
    if total == 0:
        return
    ctas = _ctas(total, n_ctas, least, problems)
    assert 1 <= ctas <= n_ctas
    assert [_begin(i, total, ctas) for i in range(ctas + 1)] == [i * total // ctas for i in range(ctas + 1)]
    held = {}
    for i in range(ctas):
        u, end = _begin(i, total, ctas), _begin(i + 1, total, ctas)
        while u < end:
            p = int(np.searchsorted(first, u, "right")) - 1
            frm, to = u - first[p], min(units[p], u - first[p] + end - u)
            t0, t1 = max(0, frm - lead), max(0, to - lead)
            if t1 > t0:
                held.setdefault(p, []).append((i, int(t0), int(t1)))
            u += to - frm
    partials = set()
    for p in range(problems):
        parts = held.get(p, [])
        assert [t for _, a, b in parts for t in range(a, b)] == list(range(tiles[p]))
        if tiles[p]:
            owner = lambda u: ((int(u) + 1) * ctas - 1) // total  # noqa: E731
            i0, i1 = owner(first[p] + lead), owner(first[p] + lead + tiles[p] - 1)
            assert [i for i, _, _ in parts] == list(range(i0, i1 + 1))
        for i, _, _ in parts:
            assert i + p not in partials and i + p < n_ctas + problems
            partials.add(i + p)


# --- the oracle's pins -------------------------------------------------------------

def _ref(rng, lens, hkv, d, page):
    n_pages = sum(-(-n // page) for n in lens) + 1
    table, at = np.full((len(lens), max(-(-n // page) for n in lens)), -1), 0
    for b, n in enumerate(lens):
        table[b, :-(-n // page)] = range(at, at + -(-n // page))
        at += -(-n // page)
    return dict(k=rng.standard_normal((n_pages, hkv, page, d)), v=rng.standard_normal((n_pages, hkv, page, d)),
                table=table, lens=np.array(lens))


def test_oracle_attention_is_softmax_attention():
    """Against torch's attention in float64 on one dense sequence with a causal chain."""
    import torch
    rng = np.random.default_rng(0)
    ref = _ref(rng, [21], 2, 8, 4)
    q, k, v = rng.standard_normal((1, 5, 6, 8)), rng.standard_normal((1, 5, 2, 8)), rng.standard_normal((1, 5, 2, 8))
    o, lse, *_ = ref_cache.attention(ref, q, k, v)
    keys = np.stack([np.concatenate([ref_cache.tokens(ref, "k", 0, h), k[0, :, h]]) for h in range(2)])
    values = np.stack([np.concatenate([ref_cache.tokens(ref, "v", 0, h), v[0, :, h]]) for h in range(2)])
    mask = np.concatenate([np.ones((5, 21), bool), np.tril(np.ones((5, 5), bool))], 1)
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x))  # noqa: E731
    want = torch.nn.functional.scaled_dot_product_attention(
        t(q[0].transpose(1, 0, 2)), t(np.repeat(keys, 3, 0)), t(np.repeat(values, 3, 0)), attn_mask=t(mask))
    np.testing.assert_allclose(o[0], want.numpy().transpose(1, 0, 2), rtol=1e-12, atol=1e-12)


def test_oracle_evidence_sums_to_the_rows():
    """A row's weights over the whole cache sum to 1; constant keys share evenly."""
    rng = np.random.default_rng(1)
    ref = _ref(rng, [13, 1], 1, 4, 4)
    q = rng.standard_normal((2, 3, 2, 4))
    _, lse, *_ = ref_cache.attention(ref, q)
    acc = ref_cache.evidence(ref, q, lse)
    for b in range(2):
        assert abs(acc[b][0].sum() - 6) < 1e-12
    ref["k"][:] = 1.0
    _, lse, *_ = ref_cache.attention(ref, q)
    np.testing.assert_allclose(ref_cache.evidence(ref, q, lse, use=np.array([[True, False, True]] * 2))[0][0], 4 / 13, rtol=1e-12)


def test_oracle_choice_by_hand():
    nan = float("nan")
    assert ref_cache.choose([5, 1, 1, 9, 1, 0, 7], 7, 4, 1, 1) == [0, 1, 3, 6]
    assert ref_cache.choose([5, 1, 1, 9, 1, 0, 7], 7, 5, 0, 0) == [0, 1, 2, 3, 6]
    assert ref_cache.choose([nan, 2, nan, -1, 3], 5, 3, 0, 0) == [1, 3, 4]
    assert ref_cache.choose([nan] * 4, 4, 2, 0, 0) == [0, 1]
    assert ref_cache.choose([1, 2], 2, 2, 0, 0) == [0, 1] and ref_cache.choose([], 0, 3, 1, 1) == []


# --- the binding's own refusals ------------------------------------------------------

def test_cache_handle_refuses_what_it_cannot_pass_on():
    """Shapes, types and strides that the handle checks (CPU tensors are refused as such)."""
    import torch

    import paper_2608_05780_gb300 as ev
    from paper_2608_05780_gb300.build import build
    build()
    x = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16)
    table, lens = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for k, v in ((x, x[:2]), (x[0], x[0]), (x, x), (x.float(), x.float())):
        with pytest.raises(ValueError):
            ev.Cache(k, v, table, lens)


def test_no_weights_of_empty_caches(fake):
    """acc_len = 0 needs no acc: an empty tensor has no address. With one it does."""
    ws = ctypes.c_void_p(None)
    empty = _cache(max_pages=0, n_pages=0, k=0, v=0, table=0)
    assert _evict(fake, ctypes.byref(ws), c=empty, n=0, acc=None) == 0
    assert _evidence(fake, ctypes.byref(ws), n=0, acc=None) == 0
    assert _evict(fake, ctypes.byref(ws), n=1, acc=None) == EINVAL and _evidence(fake, ctypes.byref(ws), n=1, acc=None) == EINVAL
    fake.evisel_free(ws)


def test_an_append_reads_its_counts_while_it_writes_the_lengths(fake):
    """lens_out over counts or src (two sequences, three tokens each): other blocks would read what was written."""
    at = lambda n: ctypes.c_void_p(FAKE + 4 * n)  # noqa: E731
    ws = ctypes.c_void_p(None)
    for lens_out, counts, src in ((4, 4, None), (5, 4, None), (4, 5, None), (4, None, 4), (9, None, 4), (4, None, 5)):
        n = fake.fake_launches()
        rc = _append(fake, ctypes.byref(ws), c=_cache(lens=FAKE + 8192), lens_out=at(lens_out),
                     counts=None if counts is None else at(counts), src=None if src is None else at(src))
        _refused(fake, rc, EINVAL, n, ws)
    for lens_out, counts, src in ((6, 4, None), (4, 6, None), (10, None, 4), (4, None, 6)):
        assert _append(fake, ctypes.byref(ws), c=_cache(lens=FAKE + 8192), lens_out=at(lens_out),
                       counts=None if counts is None else at(counts), src=None if src is None else at(src)) == 0
    fake.evisel_free(ws)
