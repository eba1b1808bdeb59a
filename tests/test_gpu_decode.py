"""The decoding-step calls against the float64 oracle (oracle/decode.py): rotation,
rotated append, beam selection, reordering, and a run of them together.

Bounds, u the rounding of the 16-bit type (2^-8 bf16, 2^-11 fp16):

  rotation  the angle comes from 32 bits of a turn that is exact modulo 1 up to |p| 2^-51 turns, rounded to fp32 (2^-25 of
            a half turn: 2^-23.3 radians); sine and cosine add 2^-24, the scale 2^-24, two products and a sum 2^-23:
            (2^-21 + |p| 2^-48) (|x1| + |x2|) + u |y|, and 2^-25 for fp16's smallest numbers
  beams     exponentials off by 2^-22 + 2^-23 |x - max| relative, of which ln V covers the mean over the row; added in
            fp32 by a lane (17 roundings, chunks of a block without loss) and a warp (6), 2^-19.4 relative at worst; the rest in
            48 bits. value: 2^-18 + 2^-22 +
            2^-23 (ln V + 1); rounded once to fp32, 2^-24 |value|
  means     fp32 sums over the stored keys: (n + 8) 2^-24 mean |k| + u |mean|
"""
import math

import numpy as np
import pytest

from cache_helpers import make_cache, tensor, u_of
from oracle import cache as ref_cache
from oracle import decode as ref

pytestmark = pytest.mark.gpu


def _types():
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _check_rotated(got, want, size, far, dtype, label=""):
    got = got.double().cpu().numpy()
    bound = (2.0 ** -21 + far * 2.0 ** -48) * size + u_of(dtype) * np.abs(want) + 2.0 ** -25
    bound = np.where(size > 0, bound, 0.0)                   # what is not rotated is copied
    err = np.abs(got - want)
    assert np.all(err <= bound), f"{label}: off by {err.max():.2e}, {np.max(err / np.maximum(bound, 1e-30)):.2f} of the bound"


def _rope(ev, d, r, interleaved, sections=None, **kw):
    freqs = ref.frequencies(r, kw.get("base", 10000.0), kw.get("factor", 1.0), kw.get("original", 0), kw.get("low_turns", 1.0),
                            kw.get("high_turns", 4.0))
    return ev.Rotary(d, r, interleaved=interleaved, sections=sections, **kw), freqs


# --- rotation ----------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,r", [(64, 16), (64, 48), (64, 64), (128, 32), (128, 112), (128, 128)])
@pytest.mark.parametrize("batch,tokens,hq,hkv", [(1, 1, 28, 4), (3, 37, 5, 3), (2, 301, 1, 1)])
def test_rotation(cuda_lib, dtype, interleaved, d, r, batch, tokens, hq, hkv):
    import torch
    ev, dtype, rng = cuda_lib, _types()[dtype], np.random.default_rng(d + r + tokens)
    rope, freqs = _rope(ev, d, r, interleaved)
    (q, qr), (k, kr) = (tensor(rng, (batch, tokens, h, d), dtype) for h in (hq, hkv))
    pos = rng.integers(0, 70000, (batch, tokens)).astype(np.int32)
    p = torch.from_numpy(pos).cuda()
    q_out, k_out = ev.evisel_rotary(rope, q, k, positions=p)
    for got, x in ((q_out, qr), (k_out, kr)):
        _check_rotated(got, *ref.rotate(x, pos, freqs, interleaved), 70000, dtype)
    back, none = ev.evisel_rotary(rope, q, positions=p, transpose=True)
    assert none is None
    _check_rotated(back, *ref.rotate(qr, pos, freqs, interleaved, transpose=True), 70000, dtype, "transposed")


@pytest.mark.parametrize("kw,far", [
    (dict(base=1e6), 1 << 20), (dict(factor=4.0), 1 << 24), (dict(factor=8.0, original=8192), 1 << 20),
    (dict(factor=32.0, original=4096, low_turns=1.0, high_turns=32.0, base=500000.0), 1 << 24), (dict(scale=0.75), 5000),
    (dict(base=10000.0), (1 << 31) - 1)])
def test_frequencies_scalings_and_far_positions(cuda_lib, kw, far):
    """Long contexts: angles of millions of radians, negative positions, every scaling."""
    import torch
    ev, rng, dtype = cuda_lib, np.random.default_rng(7), torch.float16
    scale = kw.get("scale", 1.0)
    rope, freqs = _rope(ev, 128, 128, False, **kw)
    x, xr = tensor(rng, (2, 40, 3, 128), dtype)
    pos = rng.integers(-far, far, (2, 40)).astype(np.int32)
    pos[0, :4] = (far, -far, 0, -1)
    got, _ = ev.evisel_rotary(rope, x, positions=torch.from_numpy(pos).cuda())
    want, size = ref.rotate(xr, pos, freqs, scale=scale)
    _check_rotated(got, want, size, far, dtype)


def test_own_frequencies_and_sections(cuda_lib):
    import torch
    ev, rng, dtype = cuda_lib, np.random.default_rng(8), torch.bfloat16
    freqs = np.sort(rng.uniform(-0.5, 9.0, 32))[::-1].tolist()           # more than a turn per position, and backwards
    pos = rng.integers(0, 4000, (3, 2, 19)).astype(np.int32)
    p = torch.from_numpy(pos).cuda()
    x, xr = tensor(rng, (2, 19, 6, 64), dtype)
    for sections, inter in (((8, 12, 12), False), ((0, 32, 0), True), ((0, 0, 32), False), ((31, 0, 1), True)):
        rope = ev.Rotary(64, freqs=freqs, sections=sections, interleaved=inter)
        got, _ = ev.evisel_rotary(rope, x, positions=p)
        _check_rotated(got, *ref.rotate(xr, pos, freqs, inter, sections), 4000, dtype, str(sections))
    # Each axis may be a view of its own order of sequences; `first` counts on all axes alike.
    rope = ev.Rotary(64, freqs=freqs, sections=(8, 12, 12))
    flipped = p.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(ev.evisel_rotary(rope, x, positions=flipped)[0], ev.evisel_rotary(rope, x, positions=p)[0])
    first = torch.tensor([5, -70], dtype=torch.int32, device="cuda")
    got, _ = ev.evisel_rotary(rope, x, first=first)
    count = np.array([[5], [-70]]) + np.arange(19)
    _check_rotated(got, *ref.rotate(xr, np.stack([count] * 3), freqs, False, (8, 12, 12)), 100, dtype, "first")


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_layouts(cuda_lib, interleaved):
    """[T, H, d], rows of one projection, other orders, repeated rows, results in place and where they are asked for:
    the same bits."""
    import torch
    ev, rng, dtype = cuda_lib, np.random.default_rng(9), torch.bfloat16
    rope = ev.Rotary(64, 32, interleaved=interleaved)
    rows, _ = tensor(rng, (2, 33, 20, 64), dtype)
    q, k = rows[:, :, :12], rows[:, :, 12:16]
    want_q, want_k = ev.evisel_rotary(rope, q.contiguous(), k.contiguous())
    assert torch.equal(ev.evisel_rotary(rope, q, k)[0], want_q) and torch.equal(ev.evisel_rotary(rope, q, k)[1], want_k)
    for b in range(2):                                                   # the packed form
        qb, kb = ev.evisel_rotary(rope, q[b], k[b])
        assert torch.equal(qb, want_q[b]) and torch.equal(kb, want_k[b])
        pos = torch.arange(33, dtype=torch.int32, device="cuda")
        assert torch.equal(ev.evisel_rotary(rope, q[b], positions=pos)[0], want_q[b])
    headed = q.transpose(1, 2).contiguous().transpose(1, 2)              # [B, H, T, d] in memory
    assert torch.equal(ev.evisel_rotary(rope, headed, k)[0], want_q)
    wide = torch.zeros((2, 33, 30, 64), dtype=dtype, device="cuda")
    out = wide[:, :, 3:15]
    got, _ = ev.evisel_rotary(rope, q, q_out=out)
    assert got is out and torch.equal(out, want_q) and not wide[:, :, :3].any() and not wide[:, :, 15:].any()
    one = q[:, :1].expand(-1, 33, -1, -1)                                # one token's queries at all positions
    assert torch.equal(ev.evisel_rotary(rope, one)[0], ev.evisel_rotary(rope, one.contiguous())[0])
    copy = rows.clone()
    a, b = copy[:, :, :12], copy[:, :, 12:16]
    ev.evisel_rotary(rope, a, b, q_out=a, k_out=b)                       # in place in the projection's rows
    assert torch.equal(a, want_q) and torch.equal(b, want_k) and torch.equal(copy[:, :, 16:], rows[:, :, 16:])


@pytest.mark.parametrize("interleaved,sections", [(False, None), (True, None), (False, (4, 8, 12))])
def test_transpose_is_the_gradient(cuda_lib, interleaved, sections):
    """The map is linear: its columns, from unit vectors (differences of step 1), against the rows that the transposed
    call gives; and <g, R x> = <R^T g, x> for what is rotated."""
    import torch
    ev = cuda_lib
    rope = ev.Rotary(64, 48, interleaved=interleaved, sections=sections, scale=1.25)
    eye = torch.eye(64, dtype=torch.float16, device="cuda")[None].contiguous()          # one token, 64 heads
    pos = torch.tensor([777], dtype=torch.int32, device="cuda")
    if sections:
        pos = torch.tensor([[777], [3], [41]], dtype=torch.int32, device="cuda")
    forth = ev.evisel_rotary(rope, eye, positions=pos)[0][0]             # [j]: R e_j
    back = ev.evisel_rotary(rope, eye, positions=pos, transpose=True)[0][0]
    assert torch.equal(forth, back.T)
    r = forth[:48, :48].double()
    assert (r @ r.T - 1.25 ** 2 * torch.eye(48, device="cuda", dtype=torch.float64)).abs().max() <= 4 * 2 * 1.25 ** 2 * 2.0 ** -11
    assert torch.equal(forth[48:], eye[0, 48:])


def test_rotation_past_32_bits(cuda_lib):
    """Elements beyond 2^31 of a tensor, and a token stride that passes it."""
    import torch
    ev, rng = cuda_lib, np.random.default_rng(11)
    rope, freqs = _rope(ev, 128, 128, False)
    far = (1 << 31) // 2 + 64
    pool = torch.zeros(3 * far, dtype=torch.bfloat16, device="cuda")
    x = pool.as_strided((1, 3, 2, 128), (0, far, 128, 1))
    src, xr = tensor(rng, (1, 3, 2, 128), torch.bfloat16)
    x.copy_(src)
    got, _ = ev.evisel_rotary(rope, x)
    _check_rotated(got, *ref.rotate(xr, np.arange(3)[None], freqs), 3, torch.bfloat16)
    ev.evisel_rotary(rope, x, q_out=x)
    assert torch.equal(x, got)


def test_rotation_edges(cuda_lib):
    """Nothing to do, values that are no numbers (they stay in their pair), zeros at position 0."""
    import torch
    ev = cuda_lib
    rope = ev.Rotary(64)
    empty = torch.zeros((0, 5, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert ev.evisel_rotary(rope, empty)[0].shape == empty.shape
    assert ev.evisel_rotary(rope, empty.view(5, 0, 2, 64), empty.view(5, 0, 2, 64))[1].shape == (5, 0, 2, 64)
    x = torch.randn((1, 4, 2, 64), device="cuda").to(torch.bfloat16)
    assert torch.equal(ev.evisel_rotary(rope, x[:, :1])[0], x[:, :1])    # position 0: nothing turns
    y = x.clone()
    y[0, 1, 0, 5] = float("nan")
    y[0, 2, 1, 7] = float("inf")
    a, b = ev.evisel_rotary(rope, x)[0], ev.evisel_rotary(rope, y)[0]
    other = torch.ones_like(x, dtype=torch.bool)
    other[0, 1, 0, [5, 37]] = False
    other[0, 2, 1, [7, 39]] = False
    assert torch.equal(a[other], b[other]) and b[0, 1, 0, [5, 37]].isnan().all() and not b[0, 2, 1, [7, 39]].isfinite().any()


# --- append ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,layout,d,page,interleaved,r", [
    ("bf16", "hnd", 128, 64, False, 128), ("fp16", "nhd", 64, 16, True, 32), ("bf16", "nhd", 128, 128, True, 96),
    ("fp16", "hnd", 64, 32, False, 64)])
@pytest.mark.parametrize("tokens", [1, 7, 150])
@pytest.mark.parametrize("mean", [False, True])
def test_rotated_append(cuda_lib, dtype, layout, d, page, interleaved, r, tokens, mean):
    """Every way to name tokens and positions: keys as evisel_rotary and evisel_cache_append would leave them bit by bit,
    queries too, means against float64; nothing else in the pool changes."""
    import torch
    ev, rng, dtype = cuda_lib, np.random.default_rng(tokens + d), _types()[dtype]
    lens = [0, 1, page - 1, page, 3 * page + 5]
    hkv, hq, batch = 3, 6, len(lens)
    rope = ev.Rotary(d, r, interleaved=interleaved)
    (k, _), (v, _) = (tensor(rng, (batch, tokens, hkv, d), dtype) for _ in range(2))
    q, _ = tensor(rng, (batch, tokens, hq, d), dtype)
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()  # noqa: E731
    counts = rng.integers(0, tokens + 1, batch)
    counts[-1] = tokens
    src = rng.integers(0, tokens, (batch, tokens))
    at = rng.integers(-5, 9000, (batch, tokens))
    first = rng.integers(0, 9000, batch)
    place = np.array(lens)[:, None] + np.arange(tokens)
    for kw, pos_of in ((dict(), place), (dict(positions=i32(at)), at), (dict(first=i32(first)), first[:, None] + np.arange(tokens)),
                       (dict(counts=i32(counts)), place), (dict(positions=i32(at), src=i32(src), counts=i32(counts)), at)):
        cache, _ = make_cache(rng, lens, hkv, d, page, dtype, layout, room=tokens, mean=mean, poison=False)
        plain = ev.Cache(cache.k.clone(), cache.v.clone(), cache.table, cache.lens, cache.k_mean.clone() if mean else None)
        k_rot, _ = ev.evisel_rotary(rope, k, positions=i32(pos_of))
        more = {n: kw[n] for n in ("src", "counts") if n in kw}
        want, ws = ev.evisel_cache_append(plain, k_rot, v, **more)
        got, q_out, _ = ev.evisel_cache_append_rotary(cache, rope, k, v, q=q, ws=ws, **kw)
        assert torch.equal(got, want) and torch.equal(cache.k, plain.k) and torch.equal(cache.v, plain.v)
        assert torch.equal(q_out, ev.evisel_rotary(rope, q, positions=i32(pos_of))[0])
        if mean:
            kd, table = cache.k.double().cpu().numpy(), cache.table.cpu().numpy()
            km, old = cache.k_mean.double().cpu().numpy(), plain.k_mean.double().cpu().numpy()
            touched = set()
            for b, n in enumerate(got.tolist()):
                for j in range(lens[b] // page, -(-n // page) if n > lens[b] else 0):
                    x = kd[table[b, j], :, :min(page, n - j * page)]
                    m = x.mean(1)
                    bound = (page + 8) * 2.0 ** -24 * np.abs(x).mean(1) + u_of(dtype) * np.abs(m) + 2.0 ** -25
                    assert np.all(np.abs(km[table[b, j]] - m) <= bound)
                    touched.add(int(table[b, j]))
            rest = [i for i in range(len(km)) if i not in touched]
            assert np.array_equal(km[rest], old[rest])
        assert ev.evisel_status(ws) == 0


def test_rotated_append_with_three_axes_and_strides(cuda_lib):
    """Keys, values and queries cut out of one projection, positions in time, height and width; queries in place."""
    import torch
    ev, rng, dtype = cuda_lib, np.random.default_rng(3), torch.bfloat16
    rope = ev.Rotary(128, sections=(16, 24, 24), base=1e6)
    rows, _ = tensor(rng, (2, 70, 12, 128), dtype)
    q, k, v = rows[:, :, :8], rows[:, :, 8:10], rows[:, :, 10:]
    pos = torch.from_numpy(rng.integers(0, 500, (3, 2, 70)).astype(np.int32)).cuda()
    cache, _ = make_cache(rng, [100, 0], 2, 128, 64, dtype, room=70, poison=False)
    plain = ev.Cache(cache.k.clone(), cache.v.clone(), cache.table, cache.lens)
    q_rot, k_rot = ev.evisel_rotary(rope, q, k, positions=pos)
    want, ws = ev.evisel_cache_append(plain, k_rot, v)
    mine = q.contiguous()
    got, q_out, _ = ev.evisel_cache_append_rotary(cache, rope, k, v, q=mine, q_out=mine, positions=pos, ws=ws)
    assert q_out is mine and torch.equal(mine, q_rot) and torch.equal(cache.k, plain.k) and torch.equal(cache.v, plain.v)
    assert torch.equal(got, want) and ev.evisel_status(ws) == 0


def test_rotated_append_checks_device_memory(cuda_lib):
    """Lengths, counts, sources and page ids out of range: recorded, nothing written where the table holds no page."""
    import torch
    ev, rng, dtype = cuda_lib, np.random.default_rng(4), torch.bfloat16
    rope = ev.Rotary(64)
    k, _ = tensor(rng, (2, 6, 2, 64), dtype)
    bad = dict(lens=[-1, 0], count=[7, 6], less=[-2, 6], src=[[6] * 6, [-1] * 6], page=None, far=[10 ** 9, 0])
    for what, x in bad.items():
        cache, _ = make_cache(rng, [3, 20], 2, 64, 16, dtype, room=6, poison=False)
        before, kw = cache.k.clone(), {}
        owned = cache.table[cache.table >= 0].long()
        if what in ("lens", "far"):
            cache.lens = torch.tensor(x, dtype=torch.int32, device="cuda")
        elif what in ("count", "less"):
            kw["counts"] = torch.tensor(x, dtype=torch.int32, device="cuda")
        elif what == "src":
            kw["src"] = torch.tensor(x, dtype=torch.int32, device="cuda")
        else:
            cache.table = torch.full_like(cache.table, 1 << 20)
            owned = owned[:0]
        lens, _, ws = ev.evisel_cache_append_rotary(cache, rope, k, k, **kw)
        assert ev.evisel_status(ws) == -7, what
        mine = torch.zeros(cache.k.shape[0], dtype=torch.bool, device="cuda")
        mine[owned] = True
        assert torch.equal(cache.k[~mine], before[~mine]), what


@pytest.mark.parametrize("dtype,layout,d,page,interleaved,r", [
    ("bf16", "nhd", 128, 16, False, 128), ("fp16", "hnd", 64, 16, True, 48), ("bf16", "hnd", 128, 64, True, 128)])
def test_rotated_append_of_many_pages(cuda_lib, dtype, layout, d, page, interleaved, r):
    """As many pages as the kernel needs to take two heads at a time: keys, values and means as from single heads; pages that
    are none of the pool leave everything else as it is."""
    import torch
    ev, rng, dtype = cuda_lib, np.random.default_rng(page + d), _types()[dtype]
    tokens, hkv = 480 * page + 5, 4
    rope = ev.Rotary(d, r, interleaved=interleaved)
    (k, _), (v, _) = (tensor(rng, (1, tokens, hkv, d), dtype) for _ in range(2))
    cache, _ = make_cache(rng, [page + 3], hkv, d, page, dtype, layout, room=tokens, mean=True, poison=False)
    start = {n: getattr(cache, n).clone() for n in ("k", "v", "k_mean")}
    plain = ev.Cache(cache.k.clone(), cache.v.clone(), cache.table, cache.lens, cache.k_mean.clone())
    k_rot, _ = ev.evisel_rotary(rope, k, first=cache.lens)
    want, ws = ev.evisel_cache_append(plain, k_rot, v)
    got, _, _ = ev.evisel_cache_append_rotary(cache, rope, k, v, ws=ws)
    assert torch.equal(got, want) and torch.equal(cache.k, plain.k) and torch.equal(cache.v, plain.v)
    table = cache.table[0].long()
    n, pages = int(got[0]), -(-int(got[0]) // page)
    held = torch.tensor([min(page, n - j * page) for j in range(pages)], device="cuda")
    live = (torch.arange(page, device="cuda") < held[:, None])[:, None, :, None]
    x = torch.where(live, cache.k[table[:pages]].double(), 0.0)
    m, size = x.sum(2) / held[:, None, None], x.abs().sum(2) / held[:, None, None]
    err = (cache.k_mean[table[1:pages]].double() - m[1:]).abs()
    assert bool((err <= (page + 8) * 2.0 ** -24 * size[1:] + u_of(dtype) * m[1:].abs() + 2.0 ** -25).all())
    assert torch.equal(cache.k_mean[table[0]], start["k_mean"][table[0]]) and ev.evisel_status(ws) == 0
    # Every other page is none.
    for name, x in start.items():
        getattr(cache, name).copy_(x)
    broken = cache.table.clone()
    broken[0, 1::2] = torch.tensor([-1, cache.k.shape[0], 1 << 30], dtype=torch.int32,
                                   device="cuda")[torch.arange(broken[0, 1::2].numel(), device="cuda") % 3]
    cache.table = broken
    _, _, ws = ev.evisel_cache_append_rotary(cache, rope, k, v)
    assert ev.evisel_status(ws) == -7
    lost = torch.ones(cache.k.shape[0], dtype=torch.bool, device="cuda")
    lost[table[2::2]] = False
    for name in ("k", "v", "k_mean"):
        now = getattr(cache, name)
        assert torch.equal(now[lost], start[name][lost]) 
    assert torch.equal(cache.k[table[2:pages:2]][:, :, :3], plain.k[table[2:pages:2]][:, :, :3])


def test_rotated_append_of_few_tokens_to_no_page(cuda_lib):
    """Most threads of a block have no token then: pages and means stay as they are."""
    import torch
    ev, rng, dtype = cuda_lib, np.random.default_rng(8), torch.bfloat16
    for tokens in (1, 3, 17):
        k, _ = tensor(rng, (2, tokens, 3, 128), dtype)
        cache, _ = make_cache(rng, [0, 70], 3, 128, 64, dtype, room=tokens, mean=True, poison=False)
        before = [x.clone() for x in (cache.k, cache.v, cache.k_mean)]
        cache.table = torch.where(cache.table >= 0, cache.table + 1000, cache.table)
        _, _, ws = ev.evisel_cache_append_rotary(cache, ev.Rotary(128), k, k)
        assert ev.evisel_status(ws) == -7
        for x, y in zip((cache.k, cache.v, cache.k_mean), before):
            assert torch.equal(x, y)


# --- beams -------------------------------------------------------------------------

def _check_beams(out, logits, scores, n, finished=None, eos=-1, pad=0, label=""):
    """Ranks against the oracle's values within twice the bound (both that are compared may be off), a beam's own
    order exactly; logits float64 [B, K, V]."""
    got_s, parent, token, ended = (x.cpu().numpy() for x in out[:4])
    for b in range(len(logits)):
        want = ref.continuations(logits[b], scores[b], None if finished is None else finished[b], pad)
        value = {(k, v): x for x, k, v in want}
        of_beam = {k: [v for _, kk, v in want if kk == k] for k in range(logits.shape[1])}
        e = 2.0 ** -18 + 2.0 ** -22 + 2.0 ** -23 * (math.log(logits.shape[2]) + 1)
        m, taken = min(n, len(want)), {k: 0 for k in of_beam}
        for j in range(m):
            k, v = int(parent[b, j]), int(token[b, j])
            assert (k, v) in value, f"{label} {b} {j}: {(k, v)}"
            assert of_beam[k][taken[k]] == v, f"{label} {b} {j}: beam {k} goes on with {of_beam[k][taken[k]]}, not {v}"
            taken[k] += 1
            assert abs(value[k, v] - want[j][0]) <= 2 * e, f"{label} {b} {j}: {value[k, v]} where {want[j]} stands"
            assert abs(got_s[b, j] - value[k, v]) <= e + 2.0 ** -24 * abs(value[k, v]), f"{label} {b} {j}"
            assert ended[b, j] == (v == eos or (finished is not None and bool(finished[b][k])))
        assert np.all(parent[b, m:] == -1) and np.all(token[b, m:] == -1) and np.all(np.isneginf(got_s[b, m:])) and np.all(ended[b, m:])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("batch,beams,vocab,n", [
    (1, 1, 1, 1), (1, 1, 1, 5), (2, 3, 7, 6), (1, 4, 1000, 4), (3, 5, 2049, 10), (2, 2, 50257, 64), (1, 16, 4111, 32),
    (2, 64, 301, 64), (1, 1, 152064, 17)])
def test_beam_selection(cuda_lib, dtype, batch, beams, vocab, n):
    import torch
    ev, dt, rng = cuda_lib, _types()[dtype], np.random.default_rng(vocab + n)
    x = torch.from_numpy(rng.standard_normal((batch, beams, vocab)) * 2.5).to(dt)
    scores = (-20 * rng.random((batch, beams))).astype(np.float32)
    out = ev.evisel_beam_select(x.cuda(), torch.from_numpy(scores).cuda(), n, eos=3)
    _check_beams(out, x.double().numpy(), scores, n, eos=3)
    again = ev.evisel_beam_select(x.cuda(), torch.from_numpy(scores).cuda(), n, eos=3, ws=out[4])
    assert all(torch.equal(a, b) for a, b in zip(out[:4], again[:4]))
    assert ev.evisel_status(out[4]) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_beam_rows_anywhere(cuda_lib, dtype):
    """Rows that begin at any element of a 16-byte vector, with strides of their own: numbers beside them are not read
    as theirs."""
    import torch
    ev, dt, rng = cuda_lib, _types()[dtype], np.random.default_rng(2)
    scores = (-3 * rng.random((2, 3))).astype(np.float32)
    for skew in range(9):
        for vocab in (1, 5, 8, 4097):
            pool = torch.full((skew + 6 * (vocab + 3),), 1e4, dtype=dt, device="cuda")
            x = pool[skew:].as_strided((2, 3, vocab), (3 * (vocab + 3), vocab + 3, 1))
            y = torch.from_numpy(rng.standard_normal((2, 3, vocab)) * 3).to(dt)
            x.copy_(y)
            out = ev.evisel_beam_select(x, torch.from_numpy(scores).cuda(), 6)
            _check_beams(out, y.double().numpy(), scores, 6, label=f"{skew} {vocab}")
    one = torch.randn((1, 1, 999), device="cuda").to(dt)                # one row for all beams, one for all sequences
    x = one.expand(2, 3, 999)
    out = ev.evisel_beam_select(x, torch.from_numpy(scores).cuda(), 6)
    _check_beams(out, x.double().cpu().numpy(), scores, 6, label="repeated")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [40, 3001, 20011])
@pytest.mark.parametrize("kind", ["equal", "two values", "few allowed", "one allowed", "peak", "wide"])
def test_beam_ties_and_masks(cuda_lib, dtype, vocab, kind):
    """Rows of equal logits (ties go to the lower beam and token), forbidden tokens, a row that is nearly one token."""
    import torch
    ev, dt, rng = cuda_lib, _types()[dtype], np.random.default_rng(vocab)
    batch, beams, n = 2, 3, 20
    x = rng.standard_normal((batch, beams, vocab))
    if kind == "equal":
        x[:] = -1.5
    elif kind == "two values":
        x = np.where(x > 0.5, 4.0, -2.0)
    elif kind == "few allowed":
        x = np.where(rng.random(x.shape) < 8 / vocab, x, -np.inf)
    elif kind == "one allowed":
        x[:] = -np.inf
        x[:, 0, vocab // 2] = 5.0
        x[:, 2, vocab - 1] = -3e38
    elif kind == "peak":
        x[:, :, vocab // 3] = 60.0
    else:
        x = x * 1e4
    x = torch.from_numpy(x).to(dt)
    scores = np.float32([[-1, -1, -1], [-4, -0.5, -9]])
    out = ev.evisel_beam_select(x.cuda(), torch.from_numpy(scores).cuda(), n, eos=vocab // 2)
    _check_beams(out, x.double().numpy(), scores, n, eos=vocab // 2, label=kind)
    if kind == "equal":
        m = min(n, vocab)
        assert out[1][0, :m].tolist() == [0] * m and out[2][0, :m].tolist() == list(range(m))


def test_beams_that_ended_or_never_were(cuda_lib):
    """Ended beams go on as they are; scores and rows that are no numbers give nothing; no scores: 0."""
    import torch
    ev, rng = cuda_lib, np.random.default_rng(5)
    nan, inf = float("nan"), float("inf")
    x = rng.standard_normal((7, 4, 3000)).astype(np.float32)
    x[1, 0, 7] = nan
    x[1, 2, 2999] = inf
    x[2] = -inf
    x[3, 1] = nan                       # of an ended beam: not read
    scores = np.float32(rng.uniform(-3, -1, (7, 4)))
    scores[0] = (-inf, nan, inf, -1)
    scores[4] = (-inf, -inf, nan, inf)
    scores[6, 2] = -inf
    finished = np.zeros((7, 4), bool)
    finished[3, 1] = finished[5] = finished[6, 2] = finished[6, 0] = True
    dev = [torch.from_numpy(a).cuda() for a in (x, scores, finished)]
    out = ev.evisel_beam_select(dev[0], dev[1], 8, finished=dev[2], eos=11, pad=5)
    _check_beams(out, x.astype(np.float64), scores, 8, finished, 11, 5)
    assert out[1][5].tolist()[4:] == [-1] * 4 and sorted(out[1][5].tolist()[:4]) == [0, 1, 2, 3]
    assert out[1][4].tolist() == [-1] * 8 and out[1][2].tolist() == [-1] * 8 and (out[1][1] % 2 == 1).all()
    none = ev.evisel_beam_select(dev[0][5:6], None, 3)
    _check_beams(none, x[5:6].astype(np.float64), np.zeros((1, 4)), 3)
    assert ev.evisel_beam_select(dev[0][:0], dev[1][:0], 3)[0].shape == (0, 3)


@pytest.mark.parametrize("dtype,beams,vocab,n", [
    ("bf16", 2, 300001, 1), ("fp32", 3, 150003, 2), ("fp16", 1, 700001, 3), ("bf16", 1, 32000, 64), ("fp32", 1, 20003, 50),
    ("bf16", 2, 2047, 64), ("fp16", 64, 2500, 1)])
def test_beam_blocks(cuda_lib, dtype, beams, vocab, n):
    """Blocks of several chunks, fewer blocks than continuations, a block at a row's end that is empty."""
    import torch
    ev, dt, rng = cuda_lib, _types()[dtype], np.random.default_rng(vocab)
    x = torch.from_numpy(rng.standard_normal((1, beams, vocab)) * 2.5).to(dt)
    x[0, 0, vocab - 1] = x[0, 0, vocab - 5] = x[0, beams - 1, 0] = 13.0
    scores = (-3 * rng.random((1, beams))).astype(np.float32)
    out = ev.evisel_beam_select(x.cuda(), torch.from_numpy(scores).cuda(), n)
    _check_beams(out, x.double().numpy(), scores, n)
    x[:] = 0.5                          # every block's highest is its first of very many
    scores[:] = -1
    out = ev.evisel_beam_select(x.cuda(), torch.from_numpy(scores).cuda(), n)
    m = min(n, vocab)
    assert out[1][0, :m].tolist() == [0] * m and out[2][0, :m].tolist() == list(range(m))
    assert (out[0][0, :m].double().cpu() + 1 + math.log(vocab)).abs().max() <= 2.0 ** -18 + 2.0 ** -24 * 16


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("vocab", [777, 3001, 50257])
def test_equal_beams_tie(cuda_lib, dtype, vocab):
    """Equal rows have one normaliser wherever they begin in memory: ties go to the lower beam, bit by bit."""
    import torch
    ev, dt, rng = cuda_lib, _types()[dtype], np.random.default_rng(vocab)
    row = torch.from_numpy(rng.permutation(vocab) / vocab * 60 - 30).to(dt).cuda()
    want = torch.sort(row.float(), descending=True, stable=True).indices[:4].tolist()
    for stride in (vocab, vocab + 1, vocab + 3):
        x = torch.zeros(9 * stride + 1, dtype=dt, device="cuda")[1:].as_strided((1, 9, vocab), (0, stride, 1))
        x.copy_(row)
        scores, parent, token, _, _ = ev.evisel_beam_select(x, None, 36)
        same = [[v for v, y in enumerate(row.tolist()) if y == row[w].item()] for w in want[:1]][0]
        first = [(k, v) for k in range(9) for v in same][:36]           # 16-bit logits may tie within a row too
        assert list(zip(parent[0].tolist(), token[0].tolist()))[:len(first)] == first
        assert scores[0, :len(first)].unique().numel() == 1


@pytest.mark.parametrize("level", [-3.0, -300.0, -20000.0])
def test_beam_rows_that_begin_with_forbidden_tokens(cuda_lib, level):
    """More forbidden tokens than a warp has blocks at once, and then logits far below zero."""
    import torch
    rng = np.random.default_rng(9)
    x = np.full((1, 2, 400000), -np.inf)
    x[0, 0, 300000:] = rng.standard_normal(100000) + level
    x[0, 1, ::2] = rng.standard_normal(200000) + level
    x = torch.from_numpy(x).to(torch.float32)
    scores = np.float32([[-1, -2]])
    out = cuda_lib.evisel_beam_select(x.cuda(), torch.from_numpy(scores).cuda(), 64)
    _check_beams(out, x.double().numpy(), scores, 64, label=str(level))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("far", [False, True])
def test_beam_rows_with_a_block_that_is_no_number(cuda_lib, dtype, far):
    """A NaN anywhere takes the whole row out, also where a block has nothing else and the row is far from zero."""
    import torch
    dt = _types()[dtype]
    x = torch.randn((1, 4, 9000), device="cuda")
    if far:
        x[:, :3] += 3e6
    x = x.to(dt)
    x[0, 0, 2048:4096] = float("nan")
    x[0, 1, 2048:4096] = float("-inf")
    x[0, 1, 3000] = float("nan")
    x[0, 2, 8999] = float("nan")
    out = cuda_lib.evisel_beam_select(x, None, 9)
    assert out[1][0].tolist() == [3] * 9
    _check_beams(out, x.double().cpu().numpy(), np.zeros((1, 4)), 9)


@pytest.mark.parametrize("dtype,vocab", [("bf16", 8192), ("fp16", 5001), ("fp32", 3003)])
def test_beams_of_a_batch_and_alone(cuda_lib, dtype, vocab):
    """A sequence's continuations are the same bits in a batch of two launches, in one of one launch, and by itself."""
    import torch
    ev, dt = cuda_lib, _types()[dtype]
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    x = (torch.randn((45, 5, vocab), device="cuda", generator=gen) * 3).to(dt)
    scores = -torch.rand((45, 5), device="cuda", generator=gen)
    ended = torch.rand((45, 5), device="cuda", generator=gen) < 0.2
    whole = ev.evisel_beam_select(x, scores, 12, finished=ended, eos=2)[:4]
    for first, last in ((0, 1), (7, 27), (44, 45)):
        part = ev.evisel_beam_select(x[first:last], scores[first:last].contiguous(), 12, finished=ended[first:last].contiguous(), eos=2)[:4]
        assert all(torch.equal(a[first:last], b) for a, b in zip(whole, part)), first


def test_beam_rows_past_32_bits(cuda_lib):
    """Strides of sequences and beams beyond 2^31 elements, from an odd one."""
    import torch
    rng, far = np.random.default_rng(6), (1 << 31) + 5
    pool = torch.empty(3 * far + 9000, dtype=torch.bfloat16, device="cuda")
    scores = np.float32([[-1, -2], [-0.5, -3]])
    for strides in ((2 * far, far), (far, 4096), (5, far)):
        x = pool[1:].as_strided((2, 2, 4001) if strides[0] > 5 else (1, 2, 4001), (*strides, 1))
        y = torch.from_numpy(rng.standard_normal(tuple(x.shape)) * 3).to(torch.bfloat16)
        x.copy_(y)
        out = cuda_lib.evisel_beam_select(x, torch.from_numpy(scores[:len(y)]).cuda(), 9)
        _check_beams(out, y.double().numpy(), scores, 9, label=str(strides))


def test_more_equal_blocks_than_are_listed(cuda_lib):
    import torch
    x = torch.full((2, 64, 32768), -2.0, dtype=torch.bfloat16, device="cuda")
    x[1, 63, 32767] = -1.0
    scores, parent, token, _, _ = cuda_lib.evisel_beam_select(x, None, 5)
    assert parent[0].tolist() == [0] * 5 and token[0].tolist() == [0, 1, 2, 3, 4]
    assert parent[1].tolist() == [63, 0, 0, 0, 0] and token[1].tolist() == [32767, 0, 1, 2, 3]
    assert (scores[0].double().cpu() + math.log(32768)).abs().max() <= 2.0 ** -18


@pytest.mark.parametrize("vocab", [300, 5000, 200003])
@pytest.mark.parametrize("kind", ["far above", "far below", "one block far", "across", "huge"])
def test_beam_logits_far_from_zero(cuda_lib, kind, vocab):
    """Beyond 2^20, where the exponents are formed in another way: whole rows, some of a row's blocks, chunks on both sides."""
    import torch
    ev, rng = cuda_lib, np.random.default_rng(vocab)
    x = rng.standard_normal((1, 3, vocab)) * 3
    if kind == "far above":
        x += 3e6
    elif kind == "far below":
        x[:, 1:] -= 5e7
    elif kind == "one block far":
        x[:, :, :min(vocab // 2, 1024)] -= 2e6
    elif kind == "across":
        x += 2.0 ** 20
    else:
        x *= 1e37
    x = torch.from_numpy(x).to(torch.float32)
    scores = np.float32([[-1, -2, -1.5]])
    out = ev.evisel_beam_select(x.cuda(), torch.from_numpy(scores).cuda(), 2 if vocab > 9999 else 7)
    _check_beams(out, x.double().numpy(), scores, out[0].shape[1], label=kind)


# --- reordering --------------------------------------------------------------------

def _beam_cache(rng, ev, prompts, grown, beams, hkv, d, page, dtype, layout, mean, slack=1, width=0):
    """Groups of beams that share their prompts' full pages and have pages of their own from there."""
    import torch
    n_pages = sum(n // page + beams * (-(-(n + grown + slack) // page) - n // page) for n in prompts) + 3
    order, at = rng.permutation(n_pages), 0
    ends = [-(-(n + grown + slack) // page) for n in prompts]
    table = np.full((len(prompts) * beams, max(max(ends), width)), -1, np.int32)
    for g, (n, e) in enumerate(zip(prompts, ends)):
        f = n // page
        table[g * beams:(g + 1) * beams, :f] = order[at:at + f]
        at += f
        for j in range(beams):
            table[g * beams + j, f:e] = order[at:at + e - f]
            at += e - f
    pools = [torch.from_numpy(rng.standard_normal((n_pages, hkv, page, d))).to(dtype) for _ in range(2)]
    dev = [x.transpose(1, 2).contiguous().cuda().transpose(1, 2) if layout == "nhd" else x.cuda() for x in pools]
    km = torch.from_numpy(rng.standard_normal((n_pages, hkv, d))).to(dtype).cuda() if mean else None
    lens = np.repeat(np.array(prompts) + grown, beams).astype(np.int32)
    return ev.Cache(*dev, torch.from_numpy(table).cuda(), torch.from_numpy(lens).cuda(), km)


def _numpy_cache(c):
    return dict(k=c.k.double().cpu().numpy(), v=c.v.double().cpu().numpy(), table=c.table.cpu().numpy(), lens=c.lens.cpu().numpy(),
                k_mean=None if c.k_mean is None else c.k_mean.double().cpu().numpy())


def _check_reorder(ev, cache, parent, states=()):
    import torch
    want = _numpy_cache(cache)
    table, lens, moved = ref.reorder(want, parent, [s.cpu().numpy() for s in states])
    got_table, got_lens, got_states, ws = ev.evisel_cache_reorder(cache, torch.from_numpy(parent.astype(np.int32)).cuda(), states)
    assert np.array_equal(got_table.cpu().numpy(), table) and np.array_equal(got_lens.cpu().numpy(), lens)
    for a, b in zip(got_states, moved):
        assert np.array_equal(a.cpu().numpy(), b)
    now = _numpy_cache(cache)
    assert np.array_equal(now["k"], want["k"]) and np.array_equal(now["v"], want["v"])
    assert now["k_mean"] is None or np.array_equal(now["k_mean"], want["k_mean"])
    assert ev.evisel_status(ws) == 0
    return got_table, got_lens, got_states


@pytest.mark.parametrize("beams", [1, 2, 5, 31, 32, 33, 64])
@pytest.mark.parametrize("grown,page,dtype,layout,d,mean", [
    (0, 16, "bf16", "hnd", 64, True), (5, 64, "fp16", "nhd", 128, False), (130, 128, "bf16", "nhd", 128, True)])
def test_reordering(cuda_lib, beams, grown, page, dtype, layout, d, mean):
    """Random parents, none, all the same, itself, reversed; states of every size and alignment."""
    import torch
    ev, rng, dt = cuda_lib, np.random.default_rng(beams + grown), _types()[dtype]
    prompts = [0, 1, page, 2 * page + page // 2, 37]
    batch = len(prompts) * beams
    parent = rng.integers(-1, beams, (len(prompts), beams))
    parent[0], parent[1], parent[2] = -1, beams - 1, np.arange(beams)[::-1]
    cache = _beam_cache(rng, ev, prompts, grown, beams, 2, d, page, dt, layout, mean)
    states = [torch.randint(0, 250, (batch, 3), device="cuda", dtype=torch.uint8), torch.rand((batch, 2, 4200), device="cuda"),
              torch.randint(0, 99, (batch,), device="cuda"), torch.rand((batch, 5), device="cuda"),
              torch.zeros((batch, 0), device="cuda"), torch.rand((batch, 1 + 2 * 4096), device="cuda")]
    _check_reorder(ev, cache, parent, states)


@pytest.mark.parametrize("hkv,d,page,layout", [(5, 128, 16, "nhd"), (9, 64, 16, "hnd"), (3, 64, 64, "nhd"), (1, 64, 32, "hnd")])
def test_reordering_of_heads_in_groups(cuda_lib, hkv, d, page, layout):
    """Heads that do not divide into the groups that a block copies; values and means of every head."""
    import torch
    rng = np.random.default_rng(hkv)
    cache = _beam_cache(rng, cuda_lib, [page + 5, 3 * page - 1, 7], 4, 6, hkv, d, page, torch.bfloat16, layout, True)
    _check_reorder(cuda_lib, cache, rng.integers(-1, 6, (3, 6)))


def test_reordering_again_and_again(cuda_lib):
    """Many steps of appends and reorderings: every sequence's tokens are those of its line of parents, as plain lists."""
    import torch
    ev, rng, dt = cuda_lib, np.random.default_rng(6), torch.bfloat16
    beams, page, steps, hkv = 6, 16, 60, 2
    prompts = [0, 13, 48]
    cache = _beam_cache(rng, ev, prompts, 0, beams, hkv, 64, page, dt, "hnd", True, slack=steps)
    ref0 = _numpy_cache(cache)
    lines = [[ref0["k"][ref0["table"][b, i // page], :, i % page] for i in range(ref0["lens"][b])] for b in range(len(prompts) * beams)]
    ws = ev.Workspace()
    for _ in range(steps):
        k, kr = tensor(rng, (len(lines), 1, hkv, 64), dt)
        cache.lens, _ = ev.evisel_cache_append(cache, k, k, ws=ws)
        lines = [x + [kr[b, 0]] for b, x in enumerate(lines)]
        parent = rng.integers(-1, beams, (len(prompts), beams)).astype(np.int32)
        cache.table, cache.lens, _, _ = ev.evisel_cache_reorder(cache, torch.from_numpy(parent).cuda(), ws=ws)
        lines = [lines[g * beams + (p if p >= 0 else j)] for g in range(len(prompts)) for j, p in enumerate(parent[g])]
    now = _numpy_cache(cache)
    for b, line in enumerate(lines):
        assert now["lens"][b] == len(line)
        assert np.array_equal(ref_cache.tokens(now, "k", b, 0), np.array([x[0] for x in line]))
    own = [int(now["table"][b, now["lens"][b] // page]) for b in range(len(lines))]
    assert len(set(own)) == len(own) and ev.evisel_status(ws) == 0


def test_a_prompt_fans_out(cuda_lib):
    """Empty slots beside a prompt of their group take it over, the page in progress copied into their own."""
    import torch
    ev, rng = cuda_lib, np.random.default_rng(7)
    cache = _beam_cache(rng, ev, [70, 0, 64], 0, 4, 2, 64, 32, torch.float16, "nhd", True, slack=40)
    lens = cache.lens.clone()
    lens.view(3, 4)[:, 1:] = 0
    cache.lens = lens
    table, lens, _ = _check_reorder(ev, cache, np.zeros((3, 4), int))
    assert lens.tolist() == [70] * 4 + [0] * 4 + [64] * 4


def test_reordering_checks_device_memory(cuda_lib):
    """Parents and lengths out of range, sequences without a child that are longer, pages outside the pool."""
    import torch
    ev, rng = cuda_lib, np.random.default_rng(8)
    for what in ("parent", "lens", "longer", "page"):
        cache = _beam_cache(rng, ev, [40, 40], 3, 3, 2, 64, 16, torch.bfloat16, "hnd", False, slack=20)
        before, parent = cache.k.clone(), torch.zeros((2, 3), dtype=torch.int32, device="cuda")
        lens, table = cache.lens.clone(), cache.table.clone()
        if what == "parent":
            parent[0, 1] = 3
            parent[1] = torch.tensor([0, 1, 2])
        elif what == "lens":
            lens[0] = 1 << 20
        elif what == "longer":
            lens[1] += 16
            parent[1] = torch.tensor([0, 1, 2])
        else:
            table[0, 2] = 1 << 20
            table[4, 2] = -7
        cache.lens, cache.table = lens, table
        _, _, _, ws = ev.evisel_cache_reorder(cache, parent)
        assert ev.evisel_status(ws) == -7, what
        if what == "longer":
            own = int(table[2, 2])                 # the third slot's page in progress got the copy, the second's did not
            same = [i for i in range(cache.k.shape[0]) if i != own]
            assert torch.equal(cache.k[same], before[same])
        if what == "page":
            assert torch.equal(cache.k[0], before[0]) or 0 in [int(x) for x in table.flatten()]
