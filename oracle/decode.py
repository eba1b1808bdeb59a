"""Float64 oracle of the decoding-step calls: their definitions written out, one
pair, candidate and sequence at a time. Nothing here is shared with the CUDA path.
"""
import math

import numpy as np


def frequencies(r, base=10000.0, factor=1.0, original=0.0, low=1.0, high=4.0):
    """Radians per position of the r / 2 pairs."""
    out = []
    for i in range(r // 2):
        f = base ** (-2.0 * i / r)
        if original > 0:
            g = (original * f / (2 * math.pi) - low) / (high - low)
            g = min(1.0, max(0.0, g))
            f = f * (g + (1 - g) / factor)
        else:
            f = f / factor
        out.append(f)
    return out


def rotate(x, positions, freqs, interleaved=False, sections=None, scale=1.0, transpose=False):
    """x [B, T, H, d] at positions [B, T] or [3, B, T], and size [B, T, H, d]: |x1| + |x2| of each element's pair (0
    where it is not rotated), what an implementation's error is in proportion to."""
    x = np.asarray(x, np.float64)
    half = len(freqs)
    y, size = x.copy(), np.zeros_like(x)
    for i, f in enumerate(freqs):
        axis = 0
        if sections is not None:
            axis = 0 if i < sections[0] else 1 if i < sections[0] + sections[1] else 2
        p = np.asarray(positions[axis] if sections is not None else positions, np.float64)[..., None]
        c, s = scale * np.cos(p * f), scale * np.sin(p * f)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        sign = -1.0 if transpose else 1.0
        y[..., a] = x[..., a] * c - sign * x[..., b] * s
        y[..., b] = x[..., b] * c + sign * x[..., a] * s
        size[..., a] = size[..., b] = abs(scale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, size


def continuations(logits, scores, finished=None, pad=0):
    """Every continuation (value, beam, token) of one sequence, logits [K, V], best first."""
    out = []
    for k, row in enumerate(np.asarray(logits, np.float64)):
        score = float(scores[k])
        if finished is not None and finished[k]:
            if math.isfinite(score):
                out.append((score, k, pad))
            continue
        if not math.isfinite(score) or np.isnan(row).any() or np.isposinf(row).any() or np.isneginf(row).all():
            continue
        top = row.max()
        total = math.log(math.fsum(np.exp(row - top)))
        # (x - top first: of logits near 1e38 nothing of score and total would be left)
        out += [(score + ((x - top) - total), k, v) for v, x in enumerate(row.tolist()) if x > -math.inf]
    return sorted(out, key=lambda e: (-e[0], e[1], e[2]))


def donors(parent):
    """For one group: (parent, whose pages in progress it takes) of each slot."""
    k = len(parent)
    parent = [j if p < 0 else p for j, p in enumerate(parent)]
    childless = [j for j in range(k) if j not in parent]
    out, kept = [], set()
    for j in range(k):
        if parent[j] in kept:
            out.append((parent[j], childless.pop(0)))
        else:
            kept.add(parent[j])
            out.append((parent[j], parent[j]))
    return out


def reorder(cache, parent, states=()):
    """The new table, lens and states; k, v and k_mean of ``cache`` are changed in place. cache: dict of numpy arrays
    k, v [P, hkv, page, d], table [B, n], lens [B], k_mean [P, hkv, d] or None; parent [G, K]."""
    groups, beams = parent.shape
    page, table, lens = cache["k"].shape[2], cache["table"], cache["lens"]
    new_table, new_lens = table.copy(), lens.copy()
    source = np.zeros(groups * beams, int)
    copies = []
    for g in range(groups):
        for j, (p, d) in enumerate(donors(list(parent[g]))):
            c, p, d = g * beams + j, g * beams + p, g * beams + d
            full, rest = divmod(int(lens[p]), page)
            new_table[c] = np.concatenate([table[p, :full], table[d, full:]])
            new_lens[c], source[c] = lens[p], p
            if d != p and rest:
                copies.append((table[p, full], table[d, full], rest))
    for a, b, n in copies:
        for pool in (cache["k"], cache["v"]):
            pool[b, :, :n] = pool[a, :, :n]
        if cache["k_mean"] is not None:
            cache["k_mean"][b] = cache["k_mean"][a]
    return new_table, new_lens, [s[source] for s in states]
