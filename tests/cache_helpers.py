"""Small paged caches for the tests, and the bounds their results are held to.

With u the rounding of the 16-bit type (2^-8 bf16, 2^-11 fp16) and A a row's
largest sum_d |q_d k_d| scale, a logit formed from exact 16-bit products with
fp32 sums is off by at most e = (d + 8) 2^-24 A, and 2^x by ex2.approx adds 2^-21
(its argument's rounding included):

  LSE   e + 2^-21 + 2^-22 |LSE|
  O     probabilities are rounded to 16 bits before the product with V and O once
        at the end: (u + 2 (e + 2^-21)) sum p |v| + u |O| + 2^-20 sum p |v|; in fp16
        a probability below 2^-14 of the row's largest is rounded to multiples
        of 2^-24, 2^-25 sum |v| more
  acc   a sum of exp(s - LSE): relative e + 2^-21 + 2^-22 |LSE| per row
"""
import numpy as np


def u_of(dtype):
    return 2.0 ** -8 if str(dtype).endswith("bfloat16") else 2.0 ** -11


def make_cache(rng, lens, hkv, d, page, dtype, layout="hnd", room=0, gain=1.0, spare=2, per_head=False, mean=False,
               poison=True):
    """(Cache, reference dict): random pages in a random order; slots past each length hold NaN (``poison``)."""
    import torch

    import paper_2608_05780_gb300 as ev
    lens = np.asarray(lens, np.int64)
    rows = lens.reshape(len(lens), -1)                       # [B, 1] or [B, hkv]
    need = -(-(rows + room) // page)
    max_pages = max(1, int(need.max(initial=0)))
    n_pages = int(need.sum()) + spare
    order = rng.permutation(n_pages)
    table = np.full((*rows.shape, max_pages), -1, np.int32)
    at = 0
    for i in np.ndindex(*rows.shape):
        table[i][:need[i]] = order[at:at + need[i]]
        at += need[i]
    if not per_head:
        table = table[:, 0]
    pools = []
    for g in (gain, 1.0):
        x = torch.from_numpy(rng.standard_normal((n_pages, hkv, page, d)) * g).to(dtype)
        if poison:
            for i in np.ndindex(*rows.shape):
                heads = slice(None) if not per_head else i[1]
                for j in range(need[i]):
                    x[table[i[0], i[1], j] if per_head else table[i[0], j], heads, max(0, rows[i] - j * page):] = float("nan")
        pools.append(x)
    ref = dict(k=pools[0].double().numpy(), v=pools[1].double().numpy(), table=table, lens=lens)
    dev = []
    for x in pools:
        y = x.transpose(1, 2).contiguous().cuda().transpose(1, 2) if layout == "nhd" else x.cuda()
        dev.append(y)
    km = torch.zeros((n_pages, hkv, d), dtype=dtype, device="cuda") if mean else None
    cache = ev.Cache(dev[0], dev[1], torch.from_numpy(table).cuda(), torch.from_numpy(lens.astype(np.int32)).cuda(), km)
    return cache, ref


def tensor(rng, shape, dtype, gain=1.0):
    import torch
    x = torch.from_numpy(rng.standard_normal(shape) * gain).to(dtype)
    return x.cuda(), x.double().numpy()


def tree_words(allowed):
    """int32 bit words [..., T, ceil(T / 32)] on the GPU of bool [..., T, T]."""
    import torch
    t = allowed.shape[-1]
    pad = np.zeros((*allowed.shape[:-1], -(-t // 32) * 32), np.uint64)
    pad[..., :t] = allowed
    words = (pad.reshape(*pad.shape[:-1], -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1)
    return torch.from_numpy(words.astype(np.uint32).view(np.int32)).cuda()


def random_tree(rng, batch, t):
    """Ancestor masks: a token follows one of the four before it."""
    allowed = np.zeros((batch, t, t), bool)
    for b in range(batch):
        for i in range(t):
            if i:
                allowed[b, i] = allowed[b, rng.integers(max(0, i - 4), i)]
            allowed[b, i, i] = True
    return allowed


def check_attention(o, lse, want, d, dtype, label=""):
    o_ref, lse_ref, size, values, logit = want
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    e = (d + 8) * 2.0 ** -24 * logit + 2.0 ** -21
    none = np.isneginf(lse_ref)
    assert np.array_equal(np.isneginf(lse), none), f"{label}: rows without keys"
    err = np.abs(np.where(none, 0.0, lse) - np.where(none, 0.0, lse_ref))
    bound = e + 2.0 ** -22 * np.where(none, 0.0, np.abs(lse_ref))
    assert np.all(err <= bound), f"{label}: LSE off by {err.max():.2e}, {np.max(err / bound):.2f} of the bound"
    eo = np.moveaxis(e, 0, 2)[..., None]
    u = u_of(dtype)
    bound = (u + 2 * eo + 2.0 ** -20) * size + u * np.abs(o_ref) + (2.0 ** -25 * values if u < 2.0 ** -9 else 0.0) + 1e-30
    err = np.abs(o - o_ref)
    assert np.all(np.isfinite(o)), f"{label}: non-finite O"
    assert np.all(err <= bound), f"{label}: O off by {err.max():.2e}, {np.max(err / bound):.2f} of the bound"
