"""Float64 oracle of the paged-cache calls: their definitions written out, one
sequence, head, row and token at a time.

A cache is a dict: ``k``, ``v`` float arrays [P, hkv, page, d], ``table`` [B,
max_pages] or [B, hkv, max_pages], ``lens`` [B] or [B, hkv]. Nothing here is
shared with the CUDA path.
"""
import numpy as np


def _of(x, b, h, dims):
    return x[b, h] if x.ndim == dims + 1 else x[b]


def tokens(cache, which, b, h):
    """The cached rows of one sequence and KV head, [len, d]."""
    pool = cache[which]
    page = pool.shape[2]
    n = int(_of(cache["lens"], b, h, 1))
    row = _of(cache["table"], b, h, 2)
    return np.array([pool[row[i // page], h, i % page] for i in range(n)], np.float64).reshape(n, pool.shape[3])


def attention(cache, q, k_new=None, v_new=None, allowed=None, drafted=None, scale=None):
    """O [B, T, hq, d], LSE [hq, B, T], and what bounds an implementation's error: sum p |v| [B, T, hq, d], sum |v|
    over the attended keys (the same shape) and the largest sum_d |q_d k_d| scale of a row [hq, B, T].

    allowed: bool [B, T, T] (row t attends drafted token j), None: j <= t."""
    batch, n_new, hq, d = q.shape
    hkv = cache["k"].shape[1]
    scale = 1 / np.sqrt(d) if scale is None else scale
    o, size, values = (np.zeros((batch, n_new, hq, d)) for _ in range(3))
    lse, logit = np.full((hq, batch, n_new), -np.inf), np.zeros((hq, batch, n_new))
    for b in range(batch):
        n = n_new if drafted is None else int(drafted[b])
        for h in range(hkv):
            k, v = tokens(cache, "k", b, h), tokens(cache, "v", b, h)
            for t in range(n):
                if k_new is not None:
                    js = [j for j in range(n) if (j <= t if allowed is None else allowed[b, t, j])]
                    kk = np.concatenate([k, np.float64(k_new[b, js, h]).reshape(-1, d)])
                    vv = np.concatenate([v, np.float64(v_new[b, js, h]).reshape(-1, d)])
                else:
                    kk, vv = k, v
                if not len(kk):
                    continue
                for g in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                    row = np.float64(q[b, t, g])
                    s = kk @ row * scale
                    m = s.max()
                    e = np.exp(s - m)
                    p = e / e.sum()
                    lse[g, b, t] = m + np.log(e.sum())
                    o[b, t, g] = p @ vv
                    size[b, t, g] = p @ np.abs(vv)
                    values[b, t, g] = np.abs(vv).sum(0)
                    logit[g, b, t] = (np.abs(kk) @ np.abs(row)).max() * scale
    return o, lse, size, values, logit


def evidence(cache, q, lse, use=None, drafted=None, scale=None):
    """Attention weight per cached token: a list [B][hkv] of arrays [len]."""
    batch, n_new, hq, d = q.shape
    hkv = cache["k"].shape[1]
    scale = 1 / np.sqrt(d) if scale is None else scale
    out = []
    for b in range(batch):
        out.append([])
        for h in range(hkv):
            k = tokens(cache, "k", b, h)
            acc = np.zeros(len(k))
            for t in range(n_new if drafted is None else int(drafted[b])):
                if use is not None and not use[b, t]:
                    continue
                for g in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                    if lse[g, b, t] != -np.inf:
                        acc += np.exp(k @ np.float64(q[b, t, g]) * scale - np.float64(lse[g, b, t]))
            out[-1].append(acc)
    return out


def choose(score, n, budget, sink, recent):
    """Ascending positions kept of n: all, or the first ``sink``, the last ``recent`` and the highest of the rest
    (ties to the lower position, NaN lowest)."""
    if n <= budget:
        return list(range(n))
    rest = sorted(range(sink, n - recent), key=lambda i: (np.isnan(score[i]), -score[i] if score[i] == score[i] else 0, i))
    return sorted([*range(sink), *rest[:budget - sink - recent], *range(n - recent, n)])


def page_scores(cache, k_mean, q, b, h, drafted=None):
    """max over the rows of q . k_mean per logical page of one sequence and KV head."""
    n = int(_of(cache["lens"], b, h, 1))
    page, gq = cache["k"].shape[2], q.shape[2] // cache["k"].shape[1]
    row = _of(cache["table"], b, h, 2)
    live = q.shape[1] if drafted is None else int(drafted[b])
    rows = np.float64(q[b, :live, h * gq:(h + 1) * gq]).reshape(-1, q.shape[3])
    return np.array([(rows @ np.float64(k_mean[row[j], h])).max(initial=-np.inf) for j in range(-(-n // page))])
