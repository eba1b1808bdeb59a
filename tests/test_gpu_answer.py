"""The example that runs the cache calls together, against the oracle at each step."""
import numpy as np
import pytest

from cache_helpers import check_attention
from gpu_helpers import MAP_ABS
from oracle import cache as ref_cache
from paper_2608_05780_gb300 import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,budget,page", [("tiny", 200, 16), ("single", 1024, 64)])
def test_answer_example(cuda_lib, name, budget, page):
    """The cache's evidence of the text rows is the probe's map summed over the groups' heads; the tokens kept are the
    ones that evidence ranks highest; every step's attention is exact over what the cache then holds."""
    import torch
    from paper_2608_05780_gb300.answer import answer
    probe = wl.make_probe(wl.CONFIGS[name])
    cfg, n, n_vis = probe.cfg, int(probe.cu_seqlens[1]), int(probe.n_vis[0])
    got = answer(probe, budget=budget, page=page, steps=2, drafted=5, n_select=4)
    assert got["status"] == 0 and got["accepted"] == [0, 2, 4]
    gq = cfg.hq // cfg.hkv
    tok = got["tok"].double().cpu().numpy().reshape(cfg.hkv, gq, n_vis).sum(1)
    acc = got["acc"].double().cpu().numpy()[0, :, :n]
    assert np.abs(acc[:, :n_vis] - tok).max() <= 2 * gq * MAP_ABS       # gq entries of each map
    kept = got["kept"].cpu().numpy()[0]
    weights = got["acc"].cpu().numpy()[0]
    for h in range(cfg.hkv):
        assert kept[h].tolist() == ref_cache.choose(weights[h], n, budget, cfg.tokens_per_frame, n - n_vis)

    # The cache as it stood before each step: kept tokens, then the accepted ones, all in order.
    bf = lambda x: torch.from_numpy(x).to(torch.bfloat16).double().numpy()  # noqa: E731
    k = [bf(probe.k)[kept[h], h] for h in range(cfg.hkv)]
    v = [bf(probe.v)[kept[h], h] for h in range(cfg.hkv)]
    rows, allowed = got["rows"], np.zeros((1, 5, 5), bool)
    for t in range(5):
        allowed[0, t] = [bool(rows[t] >> j & 1) for j in range(5)]
    mean = got["cache"].k_mean
    for i, s in enumerate(got["steps"]):
        m = s["lens"]
        assert m == budget + 3 * i
        pages = -(-m // page)
        pool = {x: np.zeros((pages, cfg.hkv, page, cfg.head_dim)) for x in "kv"}
        for h in range(cfg.hkv):
            for x, rows_of in (("k", k), ("v", v)):
                flat = np.zeros((pages * page, cfg.head_dim))
                flat[:m] = rows_of[h]
                pool[x][:, h] = flat.reshape(pages, page, -1)
        ref = dict(pool, table=np.arange(pages)[None], lens=np.array([m]))
        q, kd, vd = (s[x].double().cpu().numpy() for x in "qkv")
        check_attention(s["o"], s["lse"], ref_cache.attention(ref, q, kd, vd, allowed), cfg.head_dim, torch.bfloat16, f"step {i}")
        # the chosen pages: first and last among them, and the attention exact over them
        chosen = s["pages"].cpu().numpy()[0]
        n_sel = min(4, pages)
        sel = dict(pool, table=chosen[None, :, :n_sel], lens=np.zeros((1, cfg.hkv), int))
        for h in range(cfg.hkv):
            ids = chosen[h][:n_sel]
            assert ids[0] == 0 and ids[-1] == pages - 1 and np.all(np.diff(ids) > 0)
            sel["lens"][0, h] = (n_sel - 1) * page + m - (pages - 1) * page
        check_attention(s["o_sparse"], s["lse_sparse"], ref_cache.attention(sel, q, kd, vd, allowed), cfg.head_dim,
                        torch.bfloat16, f"step {i}, chosen pages")
        for h in range(cfg.hkv):
            k[h] = np.concatenate([k[h], kd[0, got["accepted"], h]])
            v[h] = np.concatenate([v[h], vd[0, got["accepted"], h]])
    # The page means at the end are those of all tokens held.
    m = budget + 6
    for h in range(cfg.hkv):
        for j in range(-(-m // page)):
            part = k[h][j * page:min(m, (j + 1) * page)]
            err = np.abs(mean[j, h].double().cpu().numpy() - part.mean(0))
            assert np.all(err <= (2.0 ** -8 + page * 2.0 ** -23) * np.abs(part).mean(0))
