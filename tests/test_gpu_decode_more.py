"""The decoding-step calls where their kernels' rarer paths run: logits that differ by less than a value's step, more blocks
than warps, prompts long enough for several passes of a warp, pages that leave the tables, device memory out of range."""
import math

import numpy as np
import pytest

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
