"""Example: from a probe's keys and values to the tokens of an answer.

    python -m paper_2608_05780_gb300.answer [workload] [steps]

The probe runs over a video and its query. Its keys and values go into a paged
cache; the text rows' attention weight per cached token (the probe's own LSE)
picks the tokens that stay; the answer then goes on over what is left, a tree of
drafted tokens per step: attention over the cache and the tree, once over all of
it and once over the pages that the queries score highest, the accepted path
appended, its weight added to what each token has. A model's projections of the
drafted tokens are stood in for by random ones, its acceptance by a fixed rule.
"""
from __future__ import annotations

import sys

import numpy as np


def empty_cache(tokens, hkv, head_dim, page, dtype, device, means=True):
    """A cache of one sequence with room for so many tokens, in pages of their own."""
    import torch

    from .cache import Cache
    n = -(-tokens // page)
    pages = [torch.zeros((n, hkv, page, head_dim), dtype=dtype, device=device) for _ in range(2)]
    table = torch.arange(n, dtype=torch.int32, device=device)[None]
    mean = torch.zeros((n, hkv, head_dim), dtype=dtype, device=device) if means else None
    return Cache(*pages, table, torch.zeros(1, dtype=torch.int32, device=device), mean)


def path_tree(tokens, device):
    """Ancestor bits of a small tree: two branches from token 0, the even and the odd tokens."""
    import torch
    rows = [1]
    for t in range(1, tokens):
        rows.append((rows[t - 2] if t > 2 else 1) | 1 << t)
    words = [[(r >> 32 * w) & 0xFFFFFFFF for w in range(-(-tokens // 32))] for r in rows]
    return torch.tensor(words, dtype=torch.int64, device=device).to(torch.int32), rows


def answer(probe, qkv=None, budget=256, steps=3, drafted=6, page=32, n_select=4, seed=0):
    """Runs the example on the first video of ``probe`` (workloads.make_probe); returns what each step computed."""
    import torch

    from . import (evisel_cache_append, evisel_cache_attention, evisel_cache_evict, evisel_cache_evidence,
                   evisel_cache_select, evisel_evidence_reduce, evisel_probe_attention, evisel_status)
    cfg = probe.cfg
    if qkv is None:
        qkv = [torch.from_numpy(x).cuda().to(torch.bfloat16) for x in (probe.q, probe.k, probe.v)]
    q, k, v = qkv
    n, n_vis = int(probe.cu_seqlens[1]), int(probe.n_vis[0])
    n_text, dev, gen = n - n_vis, q.device, torch.Generator(device=q.device).manual_seed(seed)
    out = {"steps": []}

    # The prefill, its evidence maps, and its keys and values in a cache.
    _, lse, ws = evisel_probe_attention(q, k, v, probe.cu_seqlens, probe.n_vis, cfg.tokens_per_frame, cfg.tile, probe.row_ptr,
                                        probe.col_idx)
    out["tok"], *_ = evisel_evidence_reduce(ws, cfg.hq, probe.n_vis, cfg.tokens_per_frame, len(probe.n_vis))
    full = empty_cache(n, cfg.hkv, cfg.head_dim, page, q.dtype, dev)
    full.lens, _ = evisel_cache_append(full, k[None, :n], v[None, :n], ws=ws)

    # What the text rows look at; the query itself and the first frame always stay.
    acc, _ = evisel_cache_evidence(full, q[None, n_vis:n], lse[:, n_vis:n].contiguous()[:, None], ws=ws)
    cache = empty_cache(budget + steps * drafted, cfg.hkv, cfg.head_dim, page, q.dtype, dev)
    out["acc"] = acc
    out["kept"], acc, _ = evisel_cache_evict(full, acc, cache, budget, sink=cfg.tokens_per_frame, recent=n_text, ws=ws)

    tree, rows = path_tree(drafted, dev)
    accepted = [t for t in range(drafted) if rows[drafted - 1] >> t & 1]      # the last token's branch
    src = torch.zeros((1, drafted), dtype=torch.int32, device=dev)
    src[0, :len(accepted)] = torch.tensor(accepted, dtype=torch.int32)
    counts = torch.tensor([len(accepted)], dtype=torch.int32, device=dev)
    use = torch.zeros((1, drafted), dtype=torch.bool, device=dev)
    use[0, accepted] = True
    for _ in range(steps):
        def project(heads):
            x = torch.randn((1, drafted, heads, cfg.head_dim), generator=gen, device=dev)
            return x.to(q.dtype)
        qd, kd, vd = project(cfg.hq), project(cfg.hkv), project(cfg.hkv)
        o, lse, _ = evisel_cache_attention(cache, qd, kd, vd, tree=tree, ws=ws)
        view, pages, _ = evisel_cache_select(cache, qd, n_select, sink=1, recent=1, ws=ws)
        o_sparse, lse_sparse, _ = evisel_cache_attention(view, qd, kd, vd, tree=tree, ws=ws)
        evisel_cache_evidence(cache, qd, lse, acc=acc, use=use, accumulate=True, ws=ws)
        out["steps"].append(dict(q=qd, k=kd, v=vd, o=o, lse=lse, pages=pages, o_sparse=o_sparse, lse_sparse=lse_sparse,
                                 lens=int(cache.lens[0])))
        cache.lens, _ = evisel_cache_append(cache, kd, vd, src=src, counts=counts, ws=ws)
    out.update(cache=cache, full=full, weights=acc, rows=rows, accepted=accepted, status=evisel_status(ws))
    ws.free()
    return out


def main(argv):
    from . import ensure_built
    from . import workloads as wl
    ensure_built(verbose=False)
    probe = wl.make_probe(wl.CONFIGS[argv[0] if argv else "tiny"])
    steps = int(argv[1]) if len(argv) > 1 else 3
    n = int(probe.cu_seqlens[1])
    got = answer(probe, budget=max(n // 4, int(n - probe.n_vis[0]) + probe.cfg.tokens_per_frame), steps=steps)
    kept = got["kept"][0].cpu().numpy()
    print(f"{n} tokens of the prefill, {kept.shape[1]} kept per KV head; "
          f"{np.mean(kept < int(probe.n_vis[0])):.0%} of them visual")
    for i, s in enumerate(got["steps"]):
        share = (s["lse_sparse"] - s["lse"]).exp().mean()
        print(f"step {i}: {s['lens']} cached, {s['q'].shape[1]} drafted, {len(got['accepted'])} accepted; the chosen pages and "
              f"the tree hold {float(share):.0%} of the attention")
    print(f"{int(got['cache'].lens[0])} tokens cached at the end, device status {got['status']}")


if __name__ == "__main__":
    main(sys.argv[1:])
