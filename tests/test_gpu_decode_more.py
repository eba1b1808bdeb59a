"""The decoding-step calls where their kernels' rarer paths run: logits that differ by less than a value's step, more blocks
than warps, prompts long enough for several passes of a warp, pages that leave the tables, device memory out of range."""
import math

import numpy as np
import pytest

from test_gpu_decode import _beam_cache

pytestmark = pytest.mark.gpu


def _types():
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


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
