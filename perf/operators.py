"""Cases of the operators on a paged key/value cache: what runs after the prefill, while the model answers.

  append    new tokens into the cache's pages, with the page means and the lengths: a prefill's keys and values at
            once, or the accepted ones of a drafted tree
  attend    attention of T drafted tokens of each sequence over its cache and over the drafted tokens that the
            tree's bits allow (T = 1: plain decoding)
  evidence  the attention weight that queries give to each cached token, added to what they have
  evict     the cache cut down to a budget of tokens by that weight, compacted into other pages
  sparse    the pages that each KV head's queries score highest by the page means, and the attention over them

Shapes are the ones of the package's workloads: 28 query and 4 KV heads of 128 (the 7B model whose attention they
have), 4,160 to 65,664 tokens of a video with its query; and smaller heads. Every operator runs in its plain form in
32 bits, or (``own``) as the package's entry point.
"""
import math
import random

import torch

own = False             # whether run() calls the package's operators

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
QWEN = (28, 4)


# ---------------------------------------------------------------- cases
def _case(name, op, lens, tokens, heads, d, page, dtype="bf16", layout="hnd", budget=0, sink=0, recent=0, shape=1,
          gain=1.0):
    c = dict(op=op, lens=",".join(map(str, lens)), tokens=tokens, hq=heads[0], hkv=heads[1], d=d, page=page,
             dtype=dtype, layout=layout, budget=budget, sink=sink, recent=recent, shape=shape, gain=gain)
    if name:
        c["name"] = name
    return c


def _ragged(rng, batch, longest):
    """Lengths of a batch in flight: between an eighth of the longest and the longest."""
    return [max(1, int(longest * rng.uniform(0.125, 1.0))) for _ in range(batch)]


def listed():
    rng = random.Random(11)
    return [
        # One answer token after a four-minute clip (4,160 tokens): what a single user waits for, launch by launch.
        _case("attend_clip", "attend", [4160], 1, QWEN, 128, 64),
        # A server's decoding step: 32 sequences in flight, each as far as it has come.
        _case("attend_batch", "attend", _ragged(rng, 32, 16512), 1, QWEN, 128, 64, layout="nhd"),
        # Verification of a wide drafted tree over four long videos: the matrix products are the cost.
        _case("attend_tree_long", "attend", [65664, 65601, 64000, 65664], 64, QWEN, 128, 128),
        # Odd sizes: small heads, half precision, small pages that end inside tiles, a sequence without any cache and
        # one of a single token, logits sharp enough to move the running maximum.
        _case("attend_tree_odd", "attend", [7001, 0, 1, 333, 4096, 5119], 13, (16, 8), 64, 16, dtype="fp16",
              layout="nhd", gain=4.0),
        # The weight of one decoded token of each sequence, every step.
        _case("evidence_decode", "evidence", _ragged(rng, 16, 16512), 1, QWEN, 128, 64),
        # The query's text rows over a prefilled long video: the evidence by which it is cut down before the answer.
        _case("evidence_text", "evidence", [65536], 128, QWEN, 128, 64),
        # A clip's cache cut to a quarter.
        _case("evict_clip", "evict", [4160], 0, QWEN, 128, 64, budget=1024, sink=4, recent=64),
        # Long caches cut to an eighth, into pages of the other layout.
        _case("evict_long", "evict", [65664, 65664, 50001, 65601], 0, QWEN, 128, 64, budget=8192, sink=64, recent=512,
              layout="nhd"),
        # The accepted ones of 16 drafted tokens, 32 sequences.
        _case("append_accepted", "append", _ragged(rng, 32, 16512), 16, QWEN, 128, 64, layout="nhd"),
        # A prefilled long video's keys and values into an empty cache.
        _case("append_prefill", "append", [0], 65664, QWEN, 128, 64),
        # One token of eight long sequences, each KV head reading 64 of about a thousand pages.
        _case("sparse_decode", "sparse", _ragged(rng, 7, 65664) + [65664], 1, QWEN, 128, 64, budget=64, sink=1,
              recent=2),
        # A drafted tree over two 24,704-token videos, small pages.
        _case("sparse_tree", "sparse", [24704, 24001], 24, QWEN, 128, 32, budget=128, sink=2, recent=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "evidence", "evict", "append", "sparse"])
    heads, d = rng.choice([(QWEN, 128), (QWEN, 128), ((16, 8), 64), ((32, 8), 128), ((4, 2), 64), ((16, 1), 128),
                           ((6, 2), 128)])
    page = rng.choice([16, 32, 64, 128])
    dtype, layout = rng.choice(["bf16", "bf16", "fp16"]), rng.choice(["hnd", "nhd"])
    batch = rng.choice([1, 1, 2, 3, 8, 17, 32])
    # No more than a quarter of a gigabyte of keys, so that no drawn case costs more than the largest listed one.
    most = (1 << 28) // (2 * heads[1] * d * batch)
    longest = _log_int(rng, 100, min(most, 65664 if batch <= 3 else 16512))
    lens = _ragged(rng, batch, longest)
    kw = dict(dtype=dtype, layout=layout, shape=rng.randrange(1 << 20))
    if op == "attend":
        tokens = rng.choice([1, 1, 1, 2, 5, 16, 37, 64]) if batch <= 3 else rng.choice([1, 1, 2, 5])
        return _case(None, op, lens, tokens, heads, d, page, gain=rng.choice([1.0, 1.0, 4.0]), **kw)
    if op == "evidence":
        tokens = rng.choice([1, 1, 3, 32, 101]) if batch == 1 else rng.choice([1, 1, 3])
        return _case(None, op, lens, tokens, heads, d, page, **kw)
    if op == "evict":
        recent = rng.choice([0, 1, 33])
        return _case(None, op, lens, 0, heads, d, page, budget=max(40, int(longest * rng.uniform(0.05, 0.6))),
                     sink=rng.choice([0, 4]), recent=recent, **kw)
    if op == "append":
        tokens = rng.choice([1, 4, 31, 64]) if batch > 3 else _log_int(rng, 1, 20000)
        return _case(None, op, lens, tokens, heads, d, page, **kw)
    return _case(None, op, lens, rng.choice([1, 1, 4, 24]) if batch <= 3 else 1, heads, d, page,
                 budget=rng.choice([8, 33, 64]), sink=rng.choice([0, 1]), recent=rng.choice([1, 3]), **kw)


# ---------------------------------------------------------------- inputs
def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def _accepted(case):
    """Per sequence the drafted tokens that an append takes, in order: all of one run, or a path of the tree."""
    rng, tokens = random.Random(case["shape"]), case["tokens"]
    if tokens > 64:
        return [list(range(tokens)) for _ in _lens(case)]
    return [sorted(rng.sample(range(tokens), rng.randint(1, min(tokens, 8)))) for _ in _lens(case)]


def _tree(case):
    """Ancestor bits [B][T] of a random tree per sequence (a token follows one of the four before it), and how many
    tokens each sequence has drafted."""
    rng, tokens = random.Random(case["shape"]), case["tokens"]
    bits, drafted = [], []
    for _ in _lens(case):
        row = []
        for t in range(tokens):
            parent = rng.randrange(max(0, t - 4), t) if t else None
            row.append((row[parent] if parent is not None else 0) | 1 << t)
        bits.append(row)
        drafted.append(tokens if tokens == 1 else rng.randint((tokens + 1) // 2, tokens))
    return bits, drafted


def _grid(x):
    """Rounded to sixteenths within 8: products and sums of such numbers are exact in 32 bits in any order, so that a
    choice by them does not hang on the order of a sum."""
    return (x * 16).round().clamp(-128, 128) / 16


def _words(bits, tokens):
    n = -(-tokens // 32)
    rows = [[[(b >> 32 * w) & 0xFFFFFFFF for w in range(n)] for b in row] for row in bits]
    return torch.tensor(rows, dtype=torch.int64, device="cuda").to(torch.int32)


def _pool(n_pages, case, gen, fill=True):
    """Pages [P, Hkv, page, d]: with the heads outside ("hnd"), or inside the tokens ("nhd")."""
    shape = (n_pages, case["hkv"], case["page"], case["d"])
    swap = case["layout"] == "nhd"
    if swap:
        shape = (shape[0], shape[2], shape[1], shape[3])
    make = torch.randn if fill else torch.zeros
    x = make(shape, device="cuda", **(dict(generator=gen) if fill else {})).to(DTYPES[case["dtype"]])
    return x.transpose(1, 2) if swap else x


def _cache(case, lens, room, gen, fill=True):
    """Pages of a pool in a random order, ``room`` tokens more than each length, and the table of them."""
    page = case["page"]
    need = [-(-(n + room) // page) for n in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return dict(k=_pool(n_pages, case, gen, fill), v=_pool(n_pages, case, gen, fill), table=table,
                lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), k_mean=None)


def _clustered(case, c, q, gen):
    """Pages about topics of their own, and queries aimed at eight pages of their sequence: attention concentrated on
    a small share of the cache, the regime that a selection is made for. Returns queries and page means on the grid."""
    n_pages, hkv, gq = c["k"].shape[0], case["hkv"], case["hq"] // case["hkv"]
    topic = torch.randn((n_pages, hkv, case["d"]), generator=gen, device="cuda")
    c["k"] += (3 * topic)[:, :, None].to(c["k"].dtype)
    pages = ((c["lens"] + case["page"] - 1) // case["page"]).clamp(min=1)
    pick = (torch.rand((len(pages), 8), generator=gen, device="cuda") * pages[:, None]).long()
    aim = topic[c["table"].gather(1, pick).long()].sum(1) / math.sqrt(8)
    q = 0.25 * q + aim.repeat_interleave(gq, 1)[:, None]
    return _grid(q), _grid(c["k"].float().mean(2)).to(c["k"].dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed & 0x7FFFFFFFFFFF)
    lens, tokens, dtype, op = _lens(case), case["tokens"], DTYPES[case["dtype"]], case["op"]
    batch, hq, hkv, d = len(lens), case["hq"], case["hkv"], case["d"]
    s = dict(case=case, cache=_cache(case, lens, tokens if op == "append" else 0, gen))
    c = s["cache"]

    def rand(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if op in ("attend", "sparse"):
        q = rand(batch, tokens, hq, d) * case["gain"]
        if op == "sparse":
            q, c["k_mean"] = _clustered(case, c, q, gen)
        bits, drafted = _tree(case)
        s.update(q=q.to(dtype), k_new=rand(batch, tokens, hkv, d).to(dtype), v_new=rand(batch, tokens, hkv, d).to(dtype),
                 tree=_words(bits, tokens), drafted=torch.tensor(drafted, dtype=torch.int32, device="cuda"))
    elif op == "evidence":
        s["q"] = rand(batch, tokens, hq, d).to(dtype)
        rng = random.Random(case["shape"])
        s["use"] = torch.tensor([[tokens == 1 or rng.random() < 0.9 for _ in range(tokens)] for _ in lens], device="cuda")
        # Row normalisers near the ones of unit logits: half a nat above ln len, and up to one for tokens not cached.
        ln = torch.log(c["lens"].clamp(min=1).float())
        s["lse"] = (ln[None, :, None] + 0.5 + torch.rand((hq, batch, tokens), generator=gen, device="cuda")).contiguous()
        s["acc"] = torch.rand((batch, hkv, c["table"].shape[1] * case["page"]), generator=gen, device="cuda")
    elif op == "evict":
        # Weights fall off like a power, and a third of the tokens never had any: ties.
        w = torch.rand((batch, hkv, c["table"].shape[1] * case["page"]), generator=gen, device="cuda")
        s["acc"] = torch.where(w < 0.33, 0.0, w.pow(8))
        s["out"] = _cache(case, [0] * batch, case["budget"], gen, fill=False)
        s["out"]["k_mean"] = torch.zeros((s["out"]["k"].shape[0], hkv, d), dtype=dtype, device="cuda")
    else:
        s["k_new"], s["v_new"] = rand(batch, tokens, hkv, d).to(dtype), rand(batch, tokens, hkv, d).to(dtype)
        took = _accepted(case)
        s["counts"] = torch.tensor([len(x) for x in took], dtype=torch.int32, device="cuda")
        if tokens <= 64:
            s["src"] = torch.tensor([x + [0] * (tokens - len(x)) for x in took], dtype=torch.int32, device="cuda")
        c["k_mean"] = torch.zeros((c["k"].shape[0], hkv, d), dtype=dtype, device="cuda")
    if own:             # the handles that a program keeps: of its caches, and the workspace
        import paper_2608_05780_gb300 as ev
        s["ws"] = ev.Workspace()
        for name in ("cache", "out"):
            if name in s:
                s["own_" + name] = ev.Cache(**s[name])
    return s


# ---------------------------------------------------------------- the operators
def run(state):
    case = state["case"]
    return (_own if own else _plain)[case["op"]](state, case)


def _own_append(s, c):
    import paper_2608_05780_gb300 as ev
    cache = s["own_cache"]
    lens, _ = ev.evisel_cache_append(cache, s["k_new"], s["v_new"], src=s.get("src"), counts=s["counts"], ws=s["ws"])
    return {"k": cache.k, "v": cache.v, "k_mean": cache.k_mean, "lens": lens}


def _own_attend(s, c):
    import paper_2608_05780_gb300 as ev
    o, lse, _ = ev.evisel_cache_attention(s["own_cache"], s["q"], s["k_new"], s["v_new"], tree=s["tree"],
                                          drafted=s["drafted"], ws=s["ws"])
    return {"o": o, "lse": lse}


def _own_evidence(s, c):
    import paper_2608_05780_gb300 as ev
    acc, _ = ev.evisel_cache_evidence(s["own_cache"], s["q"], s["lse"], acc=s["acc"], use=s["use"], accumulate=True,
                                      ws=s["ws"])
    return acc


def _own_evict(s, c):
    import paper_2608_05780_gb300 as ev
    out = s["own_out"]
    kept, acc, _ = ev.evisel_cache_evict(s["own_cache"], s["acc"], out, c["budget"], sink=c["sink"],
                                         recent=c["recent"], ws=s["ws"])
    return {"kept": kept, "acc": acc, "k": out.k, "v": out.v, "k_mean": out.k_mean, "lens": out.lens}


def _own_sparse(s, c):
    import paper_2608_05780_gb300 as ev
    view, pages, _ = ev.evisel_cache_select(s["own_cache"], s["q"], c["budget"], sink=c["sink"], recent=c["recent"],
                                            ws=s["ws"])
    o, lse, _ = ev.evisel_cache_attention(view, s["q"], s["k_new"], s["v_new"], tree=s["tree"], drafted=s["drafted"],
                                          ws=s["ws"])
    return {"o": o, "lse": lse, "pages": pages}


def _gathered(pool, table):
    """The pages of ``table`` [B, Hkv, n] as tokens [B, Hkv, n page, d] in 32 bits (no page: zeros)."""
    heads = torch.arange(pool.shape[1], device=pool.device)[None, :, None]
    x = pool[table.clamp(min=0).long(), heads].float() * (table >= 0)[..., None, None]
    return x.flatten(2, 3)


def _plain_attention(s, c, table, lens):
    """Attention over the pages of table [B, Hkv, n] with lens [B, Hkv] tokens, and over the drafted tokens."""
    q, tokens, gq = s["q"].float(), c["tokens"], c["hq"] // c["hkv"]
    batch, scale = q.shape[0], 1 / math.sqrt(c["d"])
    rows = q.view(batch, tokens, c["hkv"], gq, c["d"]).permute(0, 2, 3, 1, 4).reshape(batch, c["hkv"], gq * tokens, c["d"])
    old = rows @ _gathered(s["cache"]["k"], table).transpose(2, 3) * scale
    cached = torch.arange(old.shape[3], device="cuda") < lens[..., None]
    old = old.masked_fill(~cached[:, :, None], -math.inf)
    at = torch.arange(tokens, device="cuda")
    seen = (s["tree"][:, :, (at // 32)] >> (at % 32)) & 1 > 0
    drafted = at < s["drafted"][:, None]
    seen = (seen & drafted[:, None, :] & drafted[:, :, None])[:, None, None].expand(-1, c["hkv"], gq, -1, -1).flatten(2, 3)
    new = rows @ s["k_new"].float().permute(0, 2, 3, 1) * scale
    new = new.masked_fill(~seen, -math.inf)
    live = drafted[:, None, None].expand(-1, c["hkv"], gq, -1).flatten(2, 3)
    top = torch.maximum(old.amax(3) if old.shape[3] else torch.full_like(new[..., 0], -math.inf), new.amax(3))
    shift = torch.where(top == -math.inf, 0.0, top)[..., None]
    p_old, p_new = torch.exp(old - shift), torch.exp(new - shift)
    total = p_old.sum(3) + p_new.sum(3)
    o = p_old @ _gathered(s["cache"]["v"], table) + p_new @ s["v_new"].float().transpose(1, 2)
    o = o / torch.where(total > 0, total, 1.0)[..., None]
    live = live & (total > 0)
    o = torch.where(live[..., None], o, 0.0).view(batch, c["hkv"], gq, tokens, c["d"]).permute(0, 3, 1, 2, 4)
    lse = torch.where(live, shift[..., 0] + torch.log(total), -math.inf).view(batch, c["hq"], tokens).transpose(0, 1)
    return {"o": o.reshape(batch, tokens, c["hq"], c["d"]).to(s["q"].dtype), "lse": lse.contiguous()}


def _plain_attend(s, c):
    table, lens = s["cache"]["table"], s["cache"]["lens"]
    return _plain_attention(s, c, table[:, None].expand(-1, c["hkv"], -1), lens[:, None].expand(-1, c["hkv"]))


def _plain_evidence(s, c):
    q, tokens, gq, cache = s["q"].float(), c["tokens"], c["hq"] // c["hkv"], s["cache"]
    batch = q.shape[0]
    k = _gathered(cache["k"], cache["table"][:, None].expand(-1, c["hkv"], -1))
    rows = q.view(batch, tokens, c["hkv"], gq, c["d"]).permute(0, 2, 3, 1, 4).reshape(batch, c["hkv"], gq * tokens, c["d"])
    lse = s["lse"].transpose(0, 1).reshape(batch, c["hkv"], gq * tokens, 1)
    p = torch.exp(rows @ k.transpose(2, 3) / math.sqrt(c["d"]) - lse)
    use = s["use"][:, None, None].expand(-1, c["hkv"], gq, -1).flatten(2, 3)[..., None]
    p = torch.where(use, p, 0.0).sum(2)
    cached = torch.arange(p.shape[2], device="cuda") < cache["lens"][:, None, None]
    s["acc"] += torch.where(cached, p, 0.0)
    return s["acc"]


def _ranked(score, forced, valid, n):
    """The positions of the n highest (ties to the lower position; ``forced`` ones first, others than ``valid`` never)
    in ascending order, [..., n] with the count in front and the width past it."""
    width = score.shape[-1]
    score = torch.where(forced, math.inf, torch.where(valid, score, -math.inf))
    score = torch.where(valid, score, -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices
    order = torch.nn.functional.pad(order, (0, max(0, n - width)), value=width)[..., :n]
    count = valid.sum(-1, keepdim=True).clamp(max=n)
    order = torch.where(torch.arange(n, device=score.device) < count, order, width)
    return torch.sort(order, dim=-1).values, count


def _means(pool, tokens):
    """The mean key of pages [..., page, d] with so many tokens each, rounded to the pool's type."""
    live = torch.arange(pool.shape[-2], device=pool.device) < tokens[..., None]
    total = torch.where(live[..., None], pool.float(), 0.0).sum(-2)
    return (total / tokens.clamp(min=1)[..., None]).to(pool.dtype)


def _plain_evict(s, c):
    cache, out, page, budget = s["cache"], s["out"], c["page"], c["budget"]
    at = torch.arange(s["acc"].shape[2], device="cuda")
    lens = cache["lens"][:, None, None].expand(-1, c["hkv"], -1)
    valid = at < lens
    forced = valid & ((at < c["sink"]) | (at >= lens - c["recent"]))
    kept, count = _ranked(s["acc"], forced, valid, budget)
    there = torch.arange(budget, device="cuda") < count
    src = torch.where(there, kept, 0)
    heads = torch.arange(c["hkv"], device="cuda")[None, :, None].expand_as(src)
    page_of = cache["table"][:, None].expand(-1, c["hkv"], -1).gather(2, src // page).clamp(min=0).long()
    to = torch.arange(budget, device="cuda").expand_as(src)
    to_page = out["table"][:, None].expand(-1, c["hkv"], -1).gather(2, to // page).long()
    pick = (to_page[there], heads[there], (to % page)[there])
    take = (page_of[there], heads[there], (src % page)[there])
    out["k"][pick], out["v"][pick] = cache["k"][take], cache["v"][take]
    out["lens"].copy_(count[:, 0, 0])
    slots = out["table"].clamp(min=0).long()
    held = (out["lens"][:, None] - torch.arange(slots.shape[1], device="cuda") * page).clamp(0, page)
    live = held > 0
    out["k_mean"][slots[live]] = _means(out["k"][slots], held[:, :, None].expand(-1, -1, c["hkv"]))[live]
    acc = torch.zeros((*kept.shape[:2], out["table"].shape[1] * page), device="cuda")
    acc[..., :budget] = torch.where(there, s["acc"].gather(2, src), 0.0)
    return {"kept": torch.where(there, kept, -1).to(torch.int32), "acc": acc, "k": out["k"], "v": out["v"],
            "k_mean": out["k_mean"], "lens": out["lens"]}


def _plain_append(s, c):
    cache, page = s["cache"], c["page"]
    order = torch.arange(c["tokens"], device="cuda")
    there = order < s["counts"][:, None]
    src = s["src"].long() if "src" in s else order.expand_as(there)
    pos = cache["lens"][:, None] + order
    to = cache["table"].gather(1, torch.where(there, pos // page, 0).long()).long()
    seq = torch.arange(there.shape[0], device="cuda")[:, None].expand_as(there)
    pick, take = (to[there], slice(None), (pos % page)[there].long()), (seq[there], src[there])
    cache["k"][pick], cache["v"][pick] = s["k_new"][take], s["v_new"][take]
    lens = cache["lens"] + s["counts"]
    slots = cache["table"].clamp(min=0).long()
    first = torch.arange(slots.shape[1], device="cuda") * page
    held = (lens[:, None] - first).clamp(0, page)
    fresh = (held > 0) & (first + page > cache["lens"][:, None])
    pages, held = slots[fresh], held[fresh]
    cache["k_mean"][pages] = _means(cache["k"][pages], held[:, None].expand(-1, c["hkv"]))
    return {"k": cache["k"], "v": cache["v"], "k_mean": cache["k_mean"], "lens": lens}


def _plain_sparse(s, c):
    cache, page, gq = s["cache"], c["page"], c["hq"] // c["hkv"]
    table, lens = cache["table"], cache["lens"]
    batch = table.shape[0]
    rows = s["q"].float().view(batch, c["tokens"], c["hkv"], gq, c["d"]).permute(0, 2, 1, 3, 4).flatten(2, 3)
    means = cache["k_mean"][table.clamp(min=0).long()].float().transpose(1, 2)
    score = (rows @ means.transpose(2, 3)).amax(2)
    n = (lens + page - 1) // page
    at = torch.arange(table.shape[1], device="cuda")
    valid = (at < n[:, None])[:, None].expand(-1, c["hkv"], -1)
    forced = valid & ((at < c["sink"]) | (at >= (n - c["recent"])[:, None]))[:, None]
    pages, count = _ranked(score, forced, valid, c["budget"])
    there = torch.arange(c["budget"], device="cuda") < count
    pages = torch.where(there, pages, -1)
    chosen = torch.where(there, table[:, None].expand(-1, c["hkv"], -1).gather(2, pages.clamp(min=0)), -1)
    held = torch.where(n > 0, lens - (n - 1) * page, 0)[:, None] + (count[..., 0] - 1).clamp(min=0) * page
    return {**_plain_attention(s, c, chosen, held), "pages": pages.to(torch.int32)}


_own = {"append": _own_append, "attend": _own_attend, "evidence": _own_evidence, "evict": _own_evict, "sparse": _own_sparse}
_plain = {"append": _plain_append, "attend": _plain_attend, "evidence": _plain_evidence, "evict": _plain_evict,
          "sparse": _plain_sparse}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    lens, tokens, page = _lens(case), case["tokens"], case["page"]
    hq, hkv, d, batch = case["hq"], case["hkv"], case["d"], len(lens)
    token = 2 * hkv * d                                     # bytes of one token's keys
    rows = batch * tokens * hq
    io = rows * (4 * d + 4) + 2 * batch * tokens * token    # queries, results, drafted keys and values
    if case["op"] == "attend":
        return {"bytes": 2 * token * sum(lens) + io, "flops": 4.0 * d * hq * tokens * (sum(lens) + batch * tokens / 2)}
    if case["op"] == "evidence":
        return {"bytes": (token + 8 * hkv) * sum(lens) + rows * (2 * d + 4), "flops": 2.0 * d * hq * tokens * sum(lens)}
    if case["op"] == "evict":
        kept = sum(min(n, case["budget"]) for n in lens)
        return {"bytes": 4 * hkv * sum(lens) + kept * (4 * token + 8 * hkv), "flops": 0}
    if case["op"] == "append":
        new = sum(len(x) for x in _accepted(case))
        return {"bytes": 4 * token * new, "flops": float(new * hkv * d)}
    pages = sum(-(-n // page) for n in lens)
    held = sum(min(n, case["budget"] * page) for n in lens)
    return {"bytes": token * pages + 2 * token * held + io,
            "flops": 2.0 * d * hq * tokens * pages + 4.0 * d * hq * tokens * held}


# ---------------------------------------------------------------- the same in 64 bits
def _tokens_of(pool, table_row, n, page, head):
    """The first n tokens of one sequence and head as float64 [n, d], page by page of its list."""
    ids = table_row[:-(-n // page)].long()
    return pool[ids, head].double().reshape(-1, pool.shape[3])[:n]


def _exact_attention(s, case, listing):
    """listing(b, h): the page ids and the number of tokens that (sequence, KV head) attends."""
    lens, tokens, gq = _lens(case), case["tokens"], case["hq"] // case["hkv"]
    bits, drafted = _tree(case)
    o = torch.zeros((len(lens), tokens, case["hq"], case["d"]), dtype=torch.float64, device="cuda")
    lse = torch.full((case["hq"], len(lens), tokens), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(len(lens)):
        n_new = drafted[b]
        allow = torch.tensor([[bool(bits[b][t] >> j & 1) for j in range(n_new)] for t in range(n_new)], device="cuda")
        for h in range(case["hkv"]):
            ids, n = listing(b, h)
            k = torch.cat([_tokens_of(s["cache"]["k"], ids, n, case["page"], h), s["k_new"][b, :n_new, h].double()])
            v = torch.cat([_tokens_of(s["cache"]["v"], ids, n, case["page"], h), s["v_new"][b, :n_new, h].double()])
            for g in range(h * gq, (h + 1) * gq):
                a = s["q"][b, :n_new, g].double() @ k.T / math.sqrt(case["d"])
                a[:, n:] = a[:, n:].masked_fill(~allow, -math.inf)
                lse[g, b, :n_new] = torch.logsumexp(a, 1)
                o[b, :n_new, g] = torch.softmax(a, 1) @ v
    return {"o": o, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    lens, page, hkv, tokens = _lens(case), case["page"], case["hkv"], case["tokens"]
    table = s["cache"]["table"]
    gq = case["hq"] // hkv
    if case["op"] == "attend":
        return _exact_attention(s, case, lambda b, h: (table[b], lens[b]))
    if case["op"] == "evidence":
        acc = s["acc"].double()
        for b, n in enumerate(lens):
            for g in range(case["hq"]):
                k = _tokens_of(s["cache"]["k"], table[b], n, page, g // gq)
                a = s["q"][b, :, g].double() @ k.T / math.sqrt(case["d"]) - s["lse"][g, b].double()[:, None]
                acc[b, g // gq, :n] += torch.exp(a[s["use"][b]]).sum(0)
        return acc
    if case["op"] == "sparse":
        chosen = {}
        pages = torch.full((len(lens), hkv, case["budget"]), -1, dtype=torch.int32)
        for b, n in enumerate(lens):
            count = -(-n // page)
            for h in range(hkv):
                mean = s["cache"]["k_mean"][table[b, :count].long(), h].double()
                q = s["q"][b, :, h * gq:(h + 1) * gq].double().reshape(-1, case["d"])
                score = (q @ mean.T).amax(0).tolist()
                always = [j for j in range(count) if j < case["sink"] or j >= count - case["recent"]]
                rest = sorted((j for j in range(count) if j not in set(always)), key=lambda j: (-score[j], j))
                ids = sorted(always + rest[:max(0, case["budget"] - len(always))])
                held = sum(min(page, n - j * page) for j in ids)
                chosen[b, h] = (table[b, torch.tensor(ids, device="cuda", dtype=torch.long)], held)
                pages[b, h, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
        return {**_exact_attention(s, case, lambda b, h: chosen[b, h]), "pages": pages}
    # Copies and choices of whole numbers: the page means are the only sums.
    if case["op"] == "evict":
        mean, acc = s["out"]["k_mean"].double(), torch.zeros_like(s["acc"], dtype=torch.float64)
        acc = acc[..., :1].expand(-1, -1, s["out"]["table"].shape[1] * page).clone()
        for b, n in enumerate(lens):
            always = set(range(min(n, case["sink"]))) | set(range(max(0, n - case["recent"]), n))
            for h in range(hkv):
                w = s["acc"][b, h].tolist()
                rest = sorted((i for i in range(n) if i not in always), key=lambda i: (-w[i], i))
                kept = torch.tensor(sorted([*always, *rest[:max(0, case["budget"] - len(always))]]), device="cuda")
                if n == 0:
                    continue
                acc[b, h, :len(kept)] = s["acc"][b, h, kept].double()
                k = s["cache"]["k"][table[b, kept // page].long(), h, kept % page].double()
                for j, part in enumerate(k.split(page)):
                    mean[int(s["out"]["table"][b, j]), h] = part.mean(0)
        return {"kept": None, "acc": acc, "k": None, "v": None, "k_mean": mean, "lens": None}
    k = s["cache"]["k"].clone()
    mean = s["cache"]["k_mean"].double()
    for b, (n, took) in enumerate(zip(lens, _accepted(case))):
        pos = torch.arange(n, n + len(took), device="cuda")
        k[table[b, pos // page].long(), :, pos % page] = s["k_new"][b, torch.tensor(took, device="cuda")]
        for j in range(n // page, -(-(n + len(took)) // page)):
            held = min(page, n + len(took) - j * page)
            mean[int(table[b, j])] = k[int(table[b, j])].double()[:, :held].mean(1)
    return {"k": None, "v": None, "k_mean": mean, "lens": None}
