"""The decoding-step calls where their kernels' rarer paths run: logits that differ by less than a value's step, more blocks
than warps, prompts long enough for several passes of a warp, pages that leave the tables, device memory out of range."""
import math

import numpy as np
import pytest

from cache_helpers import make_cache, tensor
from oracle import decode as ref
from test_gpu_decode import _beam_cache, _check_rotated, _rope

pytestmark = pytest.mark.gpu


def _types():
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# --- rotation ----------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d,r,interleaved,batch,tokens,hq,hkv", [
    ("bf16", 128, 128, False, 2, 2451, 28, 4), ("fp16", 128, 96, True, 1, 4901, 6, 2), ("bf16", 64, 64, False, 3, 1701, 16, 8),
    ("fp16", 64, 32, True, 1, 4869, 9, 4), ("bf16", 128, 112, True, 1, 4873, 13, 5), ("fp16", 64, 48, False, 2, 2441, 4, 2),
    ("bf16", 128, 128, False, 1, 1500, 28, 4), ("bf16", 128, 128, True, 2, 750, 13, 5), ("fp16", 64, 64, False, 1, 700, 65, 0)])
def test_rotation_of_prompts(cuda_lib, dtype, d, r, interleaved, batch, tokens, hq, hkv):
    """So many tokens that a warp has all heads of one, in several passes, or a share of them in two: forth, back, in place."""
    import torch
    ev, dtype, rng = cuda_lib, _types()[dtype], np.random.default_rng(tokens)
    rope, freqs = _rope(ev, d, r, interleaved)
    q, qr = tensor(rng, (batch, tokens, hq, d), dtype)
    k, kr = tensor(rng, (batch, tokens, hkv, d), dtype) if hkv else (None, None)
    pos = rng.integers(0, 70000, (batch, tokens)).astype(np.int32)
    p = torch.from_numpy(pos).cuda()
    for back in (False, True):
        got = ev.evisel_rotary(rope, q, k, positions=p, transpose=back)
        for y, x in zip(got, (qr, kr)):
            if x is not None:
                _check_rotated(y, *ref.rotate(x, pos, freqs, interleaved, transpose=back), 70000, dtype, f"back {back}")
    ev.evisel_rotary(rope, q, k, positions=p, transpose=True, q_out=q, k_out=k)
    assert torch.equal(q, got[0]) and (k is None or torch.equal(k, got[1]))


@pytest.mark.parametrize("tokens", [1, 37, 5000])
def test_rotation_into_the_rows_of_one_tensor(cuda_lib, tokens):
    """Queries and keys side by side, and rotated rows beside the plain ones: the same bits, and nothing else written."""
    import torch
    ev, rng, dtype = cuda_lib, np.random.default_rng(3), torch.bfloat16
    rope = ev.Rotary(64, 48)
    (q, _), (k, _) = (tensor(rng, (2, tokens, h, 64), dtype) for h in (5, 2))
    want = ev.evisel_rotary(rope, q, k)
    rows = torch.zeros((2, tokens, 9, 64), dtype=dtype, device="cuda")
    got = ev.evisel_rotary(rope, q, k, q_out=rows[:, :, :5], k_out=rows[:, :, 5:7])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(rows[:, :, :7], torch.cat(want, 2)) and not rows[:, :, 7:].any()
    rows = torch.cat([q, torch.zeros_like(q)], 2)
    ev.evisel_rotary(rope, rows[:, :, :5], q_out=rows[:, :, 5:])
    assert torch.equal(rows[:, :, :5], q) and torch.equal(rows[:, :, 5:], want[0])
    heads = torch.zeros((2, 7, tokens, 64), dtype=dtype, device="cuda").transpose(1, 2)
    ev.evisel_rotary(rope, q, k, q_out=heads[:, :, :5], k_out=heads[:, :, 5:])
    assert torch.equal(heads, torch.cat(want, 2))


# --- append ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,layout,d,page,interleaved,r,batch,tokens,hq,hkv", [
    ("bf16", "hnd", 128, 64, False, 128, 3, 1700, 28, 4), ("fp16", "nhd", 64, 16, True, 32, 2, 2500, 40, 5),
    ("bf16", "nhd", 128, 32, True, 96, 1, 1300, 21, 3)])
def test_rotated_append_of_a_prompt_with_its_queries(cuda_lib, dtype, layout, d, page, interleaved, r, batch, tokens, hq, hkv):
    """A warp then has all queries of a token, in several passes: they, keys and values as by evisel_rotary and
    evisel_cache_append, bit by bit."""
    import torch
    ev, dtype, rng = cuda_lib, _types()[dtype], np.random.default_rng(tokens)
    rope = ev.Rotary(d, r, interleaved=interleaved)
    (k, _), (v, _), (q, _) = (tensor(rng, (batch, tokens, h, d), dtype) for h in (hkv, hkv, hq))
    lens = [page + 3, 0, 5 * page][:batch]
    place = torch.from_numpy((np.array(lens)[:, None] + np.arange(tokens)).astype(np.int32)).cuda()
    at = torch.from_numpy(rng.integers(0, 9000, (batch, tokens)).astype(np.int32)).cuda()
    for kw, p in ((dict(), place), (dict(positions=at), at)):
        cache, _ = make_cache(rng, lens, hkv, d, page, dtype, layout, room=tokens, poison=False)
        plain = ev.Cache(cache.k.clone(), cache.v.clone(), cache.table, cache.lens)
        q_rot, k_rot = ev.evisel_rotary(rope, q, k, positions=p)
        want, ws = ev.evisel_cache_append(plain, k_rot, v)
        got, q_out, _ = ev.evisel_cache_append_rotary(cache, rope, k, v, q=q, ws=ws, **kw)
        assert torch.equal(got, want) and torch.equal(cache.k, plain.k) and torch.equal(cache.v, plain.v)
        assert torch.equal(q_out, q_rot) and ev.evisel_status(ws) == 0


# --- beams -------------------------------------------------------------------------

def _check_own_order(out, logits, n):
    """Of every beam, the tokens that go on are its first in the order of the logits themselves (ties: the lower token);
    a single beam gives all n of them."""
    parent, token = out[1].cpu().numpy(), out[2].cpu().numpy()
    for b, rows in enumerate(logits):
        assert len(rows) > 1 or (parent[b] == 0).sum() == min(n, np.sum(rows[0] > -np.inf))
        for k, row in enumerate(rows):
            got = token[b][parent[b] == k]
            assert got.tolist() == np.argsort(-row, kind="stable")[:len(got)].tolist(), (b, k)


@pytest.mark.parametrize("dtype,batch,beams,vocab,n,score,kind", [
    ("fp32", 1, 1, 8192, 1, -1e9, "steps"), ("fp32", 1, 1, 8192, 4, -1e9, "steps"), ("fp32", 2, 3, 50257, 9, -1e9, "steps"),
    ("fp32", 1, 4, 400001, 6, -1e9, "steps"), ("fp32", 70, 2, 8191, 5, -1e30, "steps"), ("fp32", 1, 1, 5000, 40, -1e9, "steps"),
    ("fp32", 1, 64, 16384, 5, -1e9, "level"), ("fp32", 1, 1, 16384, 3, 0.0, "tiny"), ("fp32", 3, 2, 7777, 12, 0.0, "tiny"),
    ("fp32", 1, 1, 16384, 3, 0.0, "subnormal"), ("bf16", 1, 1, 32000, 4, 0.0, "tiny"), ("bf16", 9, 5, 32001, 10, 0.0, "tiny"),
    ("bf16", 1, 64, 32768, 7, 0.0, "tiny"), ("bf16", 1, 1, 32000, 4, 0.0, "subnormal"), ("fp16", 1, 2, 32000, 6, 0.0, "subnormal")])
def test_beam_logits_closer_than_a_value_tells(cuda_lib, dtype, batch, beams, vocab, n, score, kind):
    """A large score, or logits near zero, leave less of a logit in its 48-bit value than it has: the highest ones lie in later
    blocks than others of the same value."""
    import torch
    dt, rng = _types()[dtype], np.random.default_rng(vocab + n)
    if kind in ("steps", "level"):
        x = rng.uniform(-8, 2, (batch, beams, vocab)) if kind == "steps" else np.full((batch, beams, vocab), 3.0)
        x = x.astype(np.float32)
        tops, step = 3 * n + 5, np.float32(3.0).view(np.int32)
        for b, k in np.ndindex(batch, beams):
            at = np.sort(rng.choice(vocab, tops, replace=False))
            x[b, k, at] = (step + np.arange(tops, dtype=np.int32) // 2).view(np.float32)     # higher the later, pairs of equals
        x = torch.from_numpy(x)
    else:
        least = dict(fp32=1.4e-45, bf16=9.2e-41, fp16=6.0e-8)[dtype] if kind == "subnormal" else 1e-20
        x = torch.from_numpy(np.sort(rng.integers(-100, 101, (batch, beams, vocab)), axis=2) * least).to(dt)
    scores = torch.full((batch, beams), score)
    out = cuda_lib.evisel_beam_select(x.to(dt).cuda(), scores.cuda(), n)
    _check_own_order(out, x.double().numpy(), n)
    assert cuda_lib.evisel_status(out[4]) == 0


@pytest.mark.parametrize("dtype,batch,beams,vocab,n,ended", [
    ("bf16", 200, 3, 20011, 6, 0.0), ("fp16", 200, 3, 20008, 6, 0.2), ("fp32", 90, 4, 20012, 8, 0.2), ("fp32", 90, 4, 20013, 8, 0.0),
    ("bf16", 700, 17, 1025, 17, 0.1), ("bf16", 2, 16, 152064, 16, 0.0), ("fp16", 3, 16, 152065, 32, 0.2), ("fp32", 2, 64, 20001, 40, 0.1)])
def test_beams_of_many_blocks(cuda_lib, dtype, batch, beams, vocab, n, ended):
    """More blocks than warps, which then carry on to other beams and sequences; more blocks of a sequence than its threads
    hold. Against sorted values in 64 bits, within twice the bound of test_gpu_decode; a beam's own order exactly."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    x = (torch.randn((batch, beams, vocab), device="cuda", generator=gen) * 2.5).to(_types()[dtype])
    scores = -5 * torch.rand((batch, beams), device="cuda", generator=gen)
    done = torch.rand((batch, beams), device="cuda", generator=gen) < ended
    got_s, parent, token, finished, ws = cuda_lib.evisel_beam_select(x, scores, n, finished=done, eos=3, pad=1)
    value = scores[..., None].double() + torch.log_softmax(x.double(), -1)
    value[done] = -math.inf
    value[..., 1][done] = scores[done].double()
    # (Of beams that have all ended there may be fewer than n.)
    there = torch.arange(n, device="cuda") < (value > -math.inf).sum((1, 2))[:, None]
    assert cuda_lib.evisel_status(ws) == 0 and torch.equal(parent >= 0, there) and torch.equal(token >= 0, there)
    assert bool((got_s[~there] == -math.inf).all()) and bool(finished[~there].all())
    e = 2.0 ** -18 + 2.0 ** -22 + 2.0 ** -23 * (math.log(vocab) + 1)
    k, v = parent.clamp(min=0).long(), token.clamp(min=0).long()
    mine = value.flatten(1).gather(1, k * vocab + v)
    assert bool(((mine - value.flatten(1).topk(n).values).abs() <= 2 * e)[there].all())
    assert bool(((got_s - mine).abs() <= e + 2.0 ** -24 * mine.abs())[there].all())
    assert torch.equal(finished[there], ((token == 3) | done.gather(1, k))[there])
    # The j-th of a beam's own is the j-th of its logits (so that none comes twice).
    x = x.masked_fill(done[..., None], -math.inf)
    x[..., 1][done] = 0
    order = torch.sort(x, descending=True, stable=True).indices[..., :n]
    same = parent[:, :, None] == parent[:, None, :]
    rank = (same & torch.ones((n, n), dtype=torch.bool, device="cuda").tril(-1)).sum(2)
    rows = torch.arange(batch, device="cuda")[:, None]
    assert torch.equal(order[rows, k, rank].int()[there], token[there])


# --- reordering --------------------------------------------------------------------

def test_pages_that_leave_the_tables(cuda_lib):
    """Steps over several page ends: from the page in progress on every page stays in one table of its group; the full pages
    that leave are those that only sequences without a child had, and are what the old table names and the new one does not."""
    import torch
    ev, rng, dt = cuda_lib, np.random.default_rng(12), torch.bfloat16
    beams, page, prompts, steps, left = 4, 16, [5, 16, 31], 40, 0
    cache, ws = _beam_cache(rng, ev, prompts, 0, beams, 2, 64, page, dt, "hnd", False, slack=steps), ev.Workspace()
    new = torch.zeros((len(prompts) * beams, 1, 2, 64), dtype=dt, device="cuda")
    for step in range(steps):
        cache.lens, _ = ev.evisel_cache_append(cache, new, new, ws=ws)
        old, lens = cache.table.cpu().numpy(), cache.lens.cpu().numpy()
        parent = rng.integers(-1, beams, (len(prompts), beams)).astype(np.int32)
        cache.table, cache.lens, _, _ = ev.evisel_cache_reorder(cache, torch.from_numpy(parent).cuda(), ws=ws)
        now = cache.table.cpu().numpy()
        for g in range(len(prompts)):
            rows, goes_on = slice(g * beams, (g + 1) * beams), {p if p >= 0 else j for j, p in enumerate(parent[g].tolist())}
            full = int(lens[g * beams]) // page
            a, b = old[rows], now[rows]
            own = [x[:, full:][x[:, full:] >= 0].tolist() for x in (a, b)]
            assert sorted(own[0]) == sorted(own[1]) and len(set(own[1])) == len(own[1])
            gone = set(a[a >= 0].tolist()) - set(b[b >= 0].tolist())
            lines = [set(a[j, :full].tolist()) for j in range(beams)]
            assert gone == set().union(*lines) - set().union(*(lines[j] for j in goes_on)), step
            assert not set(b[b >= 0].tolist()) - set(a[a >= 0].tolist())
            left += len(gone)
    assert left > 0 and ev.evisel_status(ws) == 0


@pytest.mark.parametrize("what", ["parent", "lens", "page"])
def test_reordering_writes_no_other_page(cuda_lib, what):
    """Parents, lengths and pages out of range: every page but those that valid copies of the other slots go to stays as it
    was, the other group's table and lengths are right."""
    import torch
    ev, rng = cuda_lib, np.random.default_rng(8)
    cache = _beam_cache(rng, ev, [40, 40], 3, 3, 2, 64, 16, torch.bfloat16, "hnd", True, slack=20)
    before = {n: getattr(cache, n).clone() for n in ("k", "v", "k_mean")}
    lens, table = cache.lens.clone(), cache.table.clone()
    own = table[:, 2].tolist()              # the pages in progress of 43 tokens
    parent = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    source = {own[4]: own[3], own[5]: own[3]}
    if what == "parent":
        parent[0] = torch.tensor([0, 3, 0])
        source[own[2]] = own[0]             # 3 counts as negative: the second slot stays
    elif what == "lens":
        lens[0] = 1 << 20
    else:
        table[0, 2], table[4, 2] = 1 << 20, -7
        del source[own[4]]
    cache.lens, cache.table = lens, table
    got_table, got_lens, _, ws = ev.evisel_cache_reorder(cache, parent)
    assert ev.evisel_status(ws) == -7
    for name, old in before.items():
        want = old.clone()
        for to, at in source.items():
            if name == "k_mean":
                want[to] = old[at]
            else:
                want[to][:, :11] = old[at][:, :11]
        now = getattr(cache, name)
        changed = [i for i in range(len(old)) if not torch.equal(now[i], want[i])]
        assert not changed, (name, changed)
    want = table[3:].clone()
    want[1:, :2] = table[3, :2]
    assert torch.equal(got_table[3:], want) and got_lens[3:].tolist() == [43] * 3
