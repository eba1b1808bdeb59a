"""Cases of the operators that a decoding step needs around the attention over the paged cache.

  rotary   the position rotation of queries and keys by themselves: before a prefill, or for drafted tokens; and by the
           transposed matrix, as for gradients or to take a rotation back
  append   new tokens into the cache's pages, their keys rotated on the way, with the step's queries rotated in the
           same call, the page means and the lengths
  beams    the highest continuations over a sequence's beams and the vocabulary, from the logits
  reorder  the beams that go on: tables that share full pages, their own copies of the page in progress, and the other
           states by sequence

Shapes are the ones of the package's workloads: 28 query and 4 KV heads of 128 (the 7B model whose attention they
have) with its vocabulary of 152,064, 4,160 to 65,664 tokens of a video with its query; and smaller heads and
vocabularies. Every operator runs in its plain form, or (``own``) as the package's entry point.
"""
import math
import random

import torch

own = False             # whether run() calls the package's operators

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
QWEN = (28, 4)


# ---------------------------------------------------------------- cases
def _rope(d, part=0, interleaved=False, sections="", base=10000.0, factor=1.0, original=0):
    """A rotation: of the first ``part`` dimensions (0: all), pairs of each axis, a scaling for long contexts."""
    return dict(d=d, part=part or d, interleaved=interleaved, sections=sections, base=base, factor=factor,
                original=original)


def _rotary(name, batch, tokens, heads, rope, dtype="bf16", far=0, layout="own", back=False, shape=1):
    c = dict(op="rotary", batch=batch, tokens=tokens, hq=heads[0], hkv=heads[1], dtype=dtype, far=far, layout=layout,
             back=back, shape=shape, **rope)
    return {**c, "name": name} if name else c


def _append(name, lens, tokens, heads, rope, page, dtype="bf16", layout="hnd", queries=True, means=True, take="all",
            shape=1):
    c = dict(op="append", lens=",".join(map(str, lens)), tokens=tokens, hq=heads[0], hkv=heads[1], page=page,
             dtype=dtype, layout=layout, queries=queries, means=means, take=take, shape=shape, **rope)
    return {**c, "name": name} if name else c


def _beams(name, batch, beams, vocab, n, dtype="bf16", ended=0.0, shape=1):
    c = dict(op="beams", batch=batch, beams=beams, vocab=vocab, n=n, dtype=dtype, ended=ended, shape=shape)
    return {**c, "name": name} if name else c


def _reorder(name, prompts, grown, beams, hkv, d, page, dtype="bf16", layout="hnd", means=True, weights=True, shape=1):
    c = dict(op="reorder", lens=",".join(map(str, prompts)), grown=grown, beams=beams, hkv=hkv, d=d, page=page,
             dtype=dtype, layout=layout, means=means, weights=weights, shape=shape)
    return {**c, "name": name} if name else c


def _ragged(rng, batch, longest):
    """Lengths of a batch in flight: between an eighth of the longest and the longest."""
    return [max(1, int(longest * rng.uniform(0.125, 1.0))) for _ in range(batch)]


def listed():
    rng = random.Random(17)
    return [
        # Six drafted tokens of one sequence: the smallest call, all launch.
        _rotary("rotary_drafted", 1, 6, QWEN, _rope(128, base=1e6), far=4160),
        # A prefilled long video before its probe: queries and keys, positions in time, height and width.
        _rotary("rotary_video", 1, 65664, QWEN, _rope(128, sections="16,24,24", base=1e6)),
        # Gradients of an interleaved, partly rotated head in half precision, scaled for long contexts and far along,
        # cut out of one projection's rows.
        _rotary("rotary_back_far", 3, 2731, (16, 8), _rope(64, part=32, interleaved=True, factor=8.0, original=8192),
                dtype="fp16", far=1 << 20, layout="fused", back=True),
        # A server's decoding step: one token of each of 32 sequences, its queries rotated in the same call.
        _append("append_step", _ragged(rng, 32, 16512), 1, QWEN, _rope(128, base=1e6), 64, layout="nhd"),
        # A prefilled long video's keys and values into an empty cache; the queries were rotated before.
        _append("append_video", [0], 65664, QWEN, _rope(128, sections="16,24,24", base=1e6), 64, queries=False),
        # The accepted ones of drafted trees: positions by depth, small pages and heads, half precision, partly rotated.
        _append("append_accepted", [7001, 0, 1, 333, 4096, 5119], 13, (16, 8), _rope(64, part=32, interleaved=True), 16,
                dtype="fp16", layout="nhd", take="some"),
        # The beams of one answer over a small vocabulary: what a single user waits for.
        _beams("beams_one", 1, 4, 32000, 4),
        # A server's step: 64 answers of eight beams, twice as many continuations so that ended ones can leave.
        _beams("beams_batch", 64, 8, 152064, 16),
        # Logits in 32 bits over an odd vocabulary, some beams ended.
        _beams("beams_odd", 7, 5, 50257, 10, dtype="fp32", ended=0.25),
        # Four beams of an answer about a four-minute clip.
        _reorder("reorder_clip", [4160], 37, 4, 4, 128, 64),
        # 16 answers of eight beams over ragged prompts, with the attention weight of each cached token.
        _reorder("reorder_batch", _ragged(rng, 16, 8256), 150, 8, 4, 128, 64, layout="nhd"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rope(rng, d):
    part = rng.choice([d, d, d // 2, d // 4, 3 * d // 4])
    sections = ""
    if rng.random() < 0.3:
        first = rng.randrange(part // 2)
        second = rng.randrange(part // 2 - first)
        sections = f"{first},{second},{part // 2 - first - second}"
    factor, original = rng.choice([(1.0, 0), (1.0, 0), (4.0, 0), (8.0, 4096), (32.0, 8192)])
    return _rope(d, part, rng.random() < 0.4, sections, rng.choice([10000.0, 500000.0, 1e6]), factor, original)


def draw(rng):
    op = rng.choice(["rotary", "append", "beams", "beams", "reorder"])
    heads, d = rng.choice([(QWEN, 128), (QWEN, 128), ((16, 8), 64), ((32, 8), 128), ((4, 2), 64), ((16, 1), 128),
                           ((6, 2), 128)])
    page = rng.choice([16, 32, 64, 128])
    dtype, layout = rng.choice(["bf16", "bf16", "fp16"]), rng.choice(["hnd", "nhd"])
    shape = rng.randrange(1 << 20)
    if op == "rotary":
        batch = rng.choice([1, 1, 2, 3, 8, 33])
        tokens = _log_int(rng, 1, min(40000, 65000 * 32 * 128 // (batch * sum(heads) * d)))
        return _rotary(None, batch, tokens, heads, _draw_rope(rng, d), dtype, rng.choice([0, 0, 70000, 1 << 20, 1 << 24]),
                       rng.choice(["own", "own", "fused"]), rng.random() < 0.3, shape)
    if op == "append":
        batch = rng.choice([1, 1, 2, 3, 8, 17, 32])
        take = rng.choice(["all", "some"])
        tokens = rng.choice([1, 1, 4, 31, 64]) if batch > 3 or take == "some" else _log_int(rng, 1, 20000)
        # No more than a quarter of a gigabyte of keys.
        longest = _log_int(rng, 100, min((1 << 28) // (2 * heads[1] * d * batch), 65664 if batch <= 3 else 16512))
        return _append(None, _ragged(rng, batch, longest), tokens, heads, _draw_rope(rng, d), page, dtype, layout,
                       rng.random() < 0.7, rng.random() < 0.6, take, shape)
    if op == "beams":
        beams = rng.choice([1, 2, 3, 4, 5, 8, 10, 16])
        vocab = _log_int(rng, 1000, 262144)
        batch = min(_log_int(rng, 1, 128), (64 * 8 * 152064) // (beams * vocab))
        kind = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        if kind == "fp32":
            batch = (batch + 1) // 2
        return _beams(None, batch, beams, vocab, rng.choice([beams, 2 * beams, 2 * beams]), kind,
                      rng.choice([0.0, 0.0, 0.3]), shape)
    beams, batch = rng.choice([2, 3, 4, 5, 8, 16]), rng.choice([1, 1, 3, 8, 16])
    longest = _log_int(rng, 16, min(16512, (1 << 28) // (2 * heads[1] * d * batch)))
    return _reorder(None, _ragged(rng, batch, longest), rng.choice([0, 1, 17, 64, 200]), beams, heads[1], d, page, dtype,
                    layout, rng.random() < 0.6, rng.random() < 0.5, shape)


# ---------------------------------------------------------------- inputs
def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def _sections(case):
    return [int(x) for x in case["sections"].split(",")] if case["sections"] else None


def _accepted(case):
    """Per sequence the new tokens that an append takes, in order: all, or a path of the drafted ones."""
    rng, tokens = random.Random(case["shape"]), case["tokens"]
    if case["take"] == "all":
        return [list(range(tokens)) for _ in _lens(case)]
    return [sorted(rng.sample(range(tokens), rng.randint(1, min(tokens, 8)))) for _ in _lens(case)]


def _parents(case):
    """Per group the beams that go on: good ones several times, others not at all; now and then a slot without any."""
    rng, beams = random.Random(case["shape"]), case["beams"]
    groups = []
    for _ in _lens(case):
        weight = [rng.expovariate(1.0) for _ in range(beams)]
        row = rng.choices(range(beams), weight, k=beams)
        groups.append([-1 if rng.random() < 0.02 else p for p in row])
    return groups


def _pool(n_pages, case, gen):
    """Pages [P, Hkv, page, d]: with the heads outside ("hnd"), or inside the tokens ("nhd")."""
    shape = (n_pages, case["hkv"], case["page"], case["d"])
    swap = case["layout"] == "nhd"
    if swap:
        shape = (shape[0], shape[2], shape[1], shape[3])
    x = torch.randn(shape, generator=gen, device="cuda").to(DTYPES[case["dtype"]])
    return x.transpose(1, 2) if swap else x


def _positions(case, first, tokens):
    """Positions of new tokens that begin at ``first`` [B]: counted up, or of three axes: time goes on by a frame of
    64 tokens, height and width say where in it a token is."""
    t = torch.arange(tokens, device="cuda")
    if not case["sections"]:
        return (first[:, None] + t).to(torch.int32)
    axes = torch.stack([t // 64, t % 64 // 8, t % 8])
    return (first[None, :, None] + axes[:, None]).to(torch.int32).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed & 0x7FFFFFFFFFFF)
    s = dict(case=case)
    _prepare[case["op"]](s, case, gen)
    if own:             # the handles that a program keeps: of its rotation, its cache, and the workspace
        import paper_2608_05780_gb300 as ev
        s["ws"] = ev.Workspace()
        if "part" in case:
            s["rope"] = ev.Rotary(case["d"], case["part"], base=case["base"], interleaved=case["interleaved"],
                                  sections=_sections(case), factor=case["factor"], original=case["original"],
                                  low_turns=1.0 if case["original"] else 0.0, high_turns=4.0 if case["original"] else 0.0)
        if "cache" in s:
            s["own_cache"] = ev.Cache(**s["cache"])
    return s


def _prepare_rotary(s, c, gen):
    batch, tokens, hq, hkv, d, dtype = c["batch"], c["tokens"], c["hq"], c["hkv"], c["d"], DTYPES[c["dtype"]]
    if c["layout"] == "fused":      # rows of one projection: queries, keys, values
        rows = torch.randn((batch, tokens, hq + 2 * hkv, d), generator=gen, device="cuda").to(dtype)
        s["q"], s["k"] = rows[:, :, :hq], rows[:, :, hq:hq + hkv]
    else:
        s["q"] = torch.randn((batch, tokens, hq, d), generator=gen, device="cuda").to(dtype)
        s["k"] = torch.randn((batch, tokens, hkv, d), generator=gen, device="cuda").to(dtype)
    first = torch.full((batch,), c["far"], device="cuda")
    if c["far"]:
        first -= torch.randint(0, c["far"] // 2, (batch,), generator=gen, device="cuda")
    s["positions"] = _positions(c, first, tokens)


def _prepare_append(s, c, gen):
    lens, tokens, page, dtype = _lens(c), c["tokens"], c["page"], DTYPES[c["dtype"]]
    batch, hq, hkv, d = len(lens), c["hq"], c["hkv"], c["d"]
    need = [-(-(n + tokens) // page) for n in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((batch, max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    mean = torch.zeros((n_pages, hkv, d), dtype=dtype, device="cuda") if c["means"] else None
    s["cache"] = dict(k=_pool(n_pages, c, gen), v=_pool(n_pages, c, gen), table=table,
                      lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), k_mean=mean)
    s["k_new"] = torch.randn((batch, tokens, hkv, d), generator=gen, device="cuda").to(dtype)
    s["v_new"] = torch.randn((batch, tokens, hkv, d), generator=gen, device="cuda").to(dtype)
    s["q"] = torch.randn((batch, tokens, hq, d), generator=gen, device="cuda").to(dtype) if c["queries"] else None
    s["positions"] = s["src"] = s["counts"] = None
    if c["take"] == "some":
        took = _accepted(c)
        s["counts"] = torch.tensor([len(x) for x in took], dtype=torch.int32, device="cuda")
        s["src"] = torch.tensor([x + [0] * (tokens - len(x)) for x in took], dtype=torch.int32, device="cuda")
    if c["sections"] or c["take"] == "some":
        # A drafted token stands as far behind the cache as it is deep in its tree; others in their order.
        deep = torch.arange(tokens, device="cuda") if c["take"] == "all" else torch.arange(tokens, device="cuda") // 2
        first = torch.tensor(lens, device="cuda")
        s["positions"] = (_positions(c, first, tokens) if c["sections"]
                          else (first[:, None] + deep).to(torch.int32).contiguous())


def _prepare_beams(s, c, gen):
    batch, beams, vocab = c["batch"], c["beams"], c["vocab"]
    x = torch.randn((batch, beams, vocab), generator=gen, device="cuda") * 1.5
    # A few dozen words stand out, as after a prefix that means something.
    likely = torch.randint(0, vocab, (batch, beams, 48), generator=gen, device="cuda")
    x.scatter_add_(2, likely, 3.0 + 4.0 * torch.rand((batch, beams, 48), generator=gen, device="cuda"))
    s["logits"] = x.to(DTYPES[c["dtype"]])
    # Summed log-probabilities of the beams so far: the best ones near one another.
    s["scores"] = -20.0 - 2.0 * torch.rand((batch, beams), generator=gen, device="cuda").sort(1).values
    rng = random.Random(c["shape"])
    ended = [[rng.random() < c["ended"] for _ in range(beams)] for _ in range(batch)]
    s["finished"] = torch.tensor(ended, device="cuda")


def _prepare_reorder(s, c, gen):
    prompts, grown, beams, page = _lens(c), c["grown"], c["beams"], c["page"]
    batch = len(prompts) * beams
    own_from = [n // page for n in prompts]
    ends = [-(-(n + grown + 1) // page) for n in prompts]
    n_pages = sum(f + beams * (e - f) for f, e in zip(own_from, ends)) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((batch, max(ends)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for g, (f, e) in enumerate(zip(own_from, ends)):
        table[g * beams:(g + 1) * beams, :f] = order[at:at + f]          # the prompt's full pages are shared
        at += f
        table[g * beams:(g + 1) * beams, f:e] = order[at:at + beams * (e - f)].view(beams, e - f)
        at += beams * (e - f)
    lens = [n + grown for n in prompts for _ in range(beams)]
    mean = None
    if c["means"]:
        mean = torch.randn((n_pages, c["hkv"], c["d"]), generator=gen, device="cuda").to(DTYPES[c["dtype"]])
    s["cache"] = dict(k=_pool(n_pages, c, gen), v=_pool(n_pages, c, gen), table=table,
                      lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), k_mean=mean)
    s["parent"] = torch.tensor(_parents(c), dtype=torch.int32, device="cuda")
    s["states"] = [torch.randint(0, 152064, (batch, grown + 1), generator=gen, device="cuda", dtype=torch.int32)]
    if c["weights"]:
        s["states"].append(torch.rand((batch, c["hkv"], max(ends) * page), generator=gen, device="cuda"))


_prepare = {"rotary": _prepare_rotary, "append": _prepare_append, "beams": _prepare_beams, "reorder": _prepare_reorder}


# ---------------------------------------------------------------- the operators
def run(state):
    case = state["case"]
    return (_own if own else _plain)[case["op"]](state, case)


def _own_rotary(s, c):
    import paper_2608_05780_gb300 as ev
    q, k = ev.evisel_rotary(s["rope"], s["q"], s["k"], positions=s["positions"], transpose=c["back"])
    return {"q": q, "k": k}


def _own_append(s, c):
    import paper_2608_05780_gb300 as ev
    cache = s["own_cache"]
    lens, q, _ = ev.evisel_cache_append_rotary(cache, s["rope"], s["k_new"], s["v_new"], q=s["q"],
                                               positions=s["positions"], src=s["src"], counts=s["counts"], ws=s["ws"])
    return {"k": cache.k, "v": cache.v, "k_mean": cache.k_mean, "lens": lens, "q": q}


def _own_beams(s, c):
    import paper_2608_05780_gb300 as ev
    scores, parent, token, finished, _ = ev.evisel_beam_select(s["logits"], s["scores"], c["n"], finished=s["finished"],
                                                               eos=2, pad=0, ws=s["ws"])
    return {"scores": scores, "parent": parent, "token": token, "finished": finished}


def _own_reorder(s, c):
    import paper_2608_05780_gb300 as ev
    cache = s["own_cache"]
    table, lens, states, _ = ev.evisel_cache_reorder(cache, s["parent"], s["states"], ws=s["ws"])
    return {"table": table, "lens": lens, "states": states, "k": cache.k, "v": cache.v, "k_mean": cache.k_mean}


def _turned(c, positions):
    """Cosines and sines [..., r / 2] of the pairs at positions [B, T] (of three axes: [3, B, T]). The angles, which far
    positions make large, in 64 bits."""
    half = c["part"] // 2
    i = torch.arange(half, device="cuda", dtype=torch.float64)
    freq = torch.exp(i * (-math.log(c["base"]) / half))
    if c["original"]:
        turns = c["original"] * freq / (2 * math.pi)
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        freq = freq * (keep + (1 - keep) / c["factor"])
    else:
        freq = freq / c["factor"]
    if c["sections"]:
        axis = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(_sections(c), device="cuda"))
        at = positions[axis].permute(1, 2, 0)
    else:
        at = positions[..., None]
    angle = at.double() * freq
    return torch.cos(angle).float(), torch.sin(angle).float()


def _plain_rotate(c, x, cos, sin, back=False):
    """x [B, T, H, d] rotated in 32 bits, rounded once."""
    r, f = c["part"], x.float()
    cos, sin = cos[:, :, None], -sin[:, :, None] if back else sin[:, :, None]
    lo, hi = (f[..., 0:r:2], f[..., 1:r:2]) if c["interleaved"] else (f[..., :r // 2], f[..., r // 2:r])
    lo, hi = lo * cos - hi * sin, hi * cos + lo * sin
    y = torch.stack([lo, hi], -1).flatten(-2) if c["interleaved"] else torch.cat([lo, hi], -1)
    return torch.cat([y.to(x.dtype), x[..., r:]], -1)


def _plain_rotary(s, c):
    cos, sin = _turned(c, s["positions"])
    return {"q": _plain_rotate(c, s["q"], cos, sin, c["back"]), "k": _plain_rotate(c, s["k"], cos, sin, c["back"])}


def _means(pool, tokens):
    """The mean key of pages [..., page, d] with so many tokens each, rounded to the pool's type."""
    live = torch.arange(pool.shape[-2], device=pool.device) < tokens[..., None]
    total = torch.where(live[..., None], pool.float(), 0.0).sum(-2)
    return (total / tokens.clamp(min=1)[..., None]).to(pool.dtype)


def _plain_append(s, c):
    cache, page, tokens = s["cache"], c["page"], c["tokens"]
    order = torch.arange(tokens, device="cuda")
    positions = s["positions"] if s["positions"] is not None else cache["lens"][:, None] + order
    cos, sin = _turned(c, positions)
    k_new = _plain_rotate(c, s["k_new"], cos, sin)
    counts = s["counts"] if s["counts"] is not None else torch.full_like(cache["lens"], tokens)
    there = order < counts[:, None]
    src = s["src"].long() if s["src"] is not None else order.expand_as(there)
    pos = cache["lens"][:, None] + order
    to = cache["table"].gather(1, torch.where(there, pos // page, 0).long()).long()
    seq = torch.arange(there.shape[0], device="cuda")[:, None].expand_as(there)
    pick, take = (to[there], slice(None), (pos % page)[there].long()), (seq[there], src[there])
    cache["k"][pick], cache["v"][pick] = k_new[take], s["v_new"][take]
    lens = cache["lens"] + counts
    if c["means"]:
        slots = cache["table"].clamp(min=0).long()
        first = torch.arange(slots.shape[1], device="cuda") * page
        held = (lens[:, None] - first).clamp(0, page)
        fresh = (held > 0) & (first + page > cache["lens"][:, None])
        pages, held = slots[fresh], held[fresh]
        cache["k_mean"][pages] = _means(cache["k"][pages], held[:, None].expand(-1, c["hkv"]))
    q = _plain_rotate(c, s["q"], cos, sin) if c["queries"] else None
    return {"k": cache["k"], "v": cache["v"], "k_mean": cache["k_mean"], "lens": lens, "q": q}


def _plain_beams(s, c):
    batch, beams, vocab, n = c["batch"], c["beams"], c["vocab"], c["n"]
    # In 64 bits: which of two near values is the higher one decides a token.
    x = s["logits"].double()
    top = x.amax(2, keepdim=True)
    value = x - (top + torch.log(torch.exp(x - top).sum(2, keepdim=True))) + s["scores"].double()[..., None]
    ended = s["finished"][..., None]
    value = torch.where(ended, -math.inf, value)
    value[..., 0] = torch.where(s["finished"], s["scores"].double(), value[..., 0])      # an ended beam goes on as it is
    best, at = torch.sort(value.flatten(1), dim=1, descending=True, stable=True)
    best, at = best[:, :n], at[:, :n]
    parent, token = at // vocab, at % vocab
    finished = s["finished"].gather(1, parent) | (token == 2)
    none = best == -math.inf
    return {"scores": best.float(), "parent": torch.where(none, -1, parent).to(torch.int32),
            "token": torch.where(none, -1, token).to(torch.int32), "finished": finished | none}


def _plain_reorder(s, c):
    cache, page, beams = s["cache"], c["page"], c["beams"]
    groups = s["parent"].shape[0]
    slot = torch.arange(beams, device="cuda").expand(groups, beams)
    parent = torch.where(s["parent"] < 0, slot, s["parent"].long())
    # The first child of a beam keeps the page in progress; the others, in order, take those of the beams without any.
    same = parent[:, :, None] == parent[:, None, :]
    first = ~(same & (slot[:, None, :] < slot[:, :, None])).any(2)
    childless = ~(parent[:, :, None] == slot[:, None, :]).any(1)
    free = torch.sort(torch.where(childless, slot, beams), dim=1).values
    rank = (~first).cumsum(1) - 1
    donor = torch.where(first, parent, free.gather(1, rank.clamp(min=0)))
    base = torch.arange(groups, device="cuda")[:, None] * beams
    parent, donor = (parent + base).flatten(), (donor + base).flatten()
    lens = cache["lens"][parent]
    full = lens // page
    column = torch.arange(cache["table"].shape[1], device="cuda")
    table = torch.where(column < full[:, None], cache["table"][parent], cache["table"][donor])
    copy = ((donor != parent) & (lens % page > 0)).nonzero()[:, 0]
    at = full[copy][:, None].long()
    to, fro = cache["table"][donor[copy]].gather(1, at)[:, 0].long(), cache["table"][parent[copy]].gather(1, at)[:, 0].long()
    live = (torch.arange(page, device="cuda") < (lens % page)[copy][:, None])[:, None, :, None]
    for pool in (cache["k"], cache["v"]):
        pool[to] = torch.where(live, pool[fro], pool[to])
    if c["means"]:
        cache["k_mean"][to] = cache["k_mean"][fro]
    return {"table": table, "lens": lens, "states": [x[parent] for x in s["states"]], "k": cache["k"], "v": cache["v"],
            "k_mean": cache["k_mean"]}


_own = {"rotary": _own_rotary, "append": _own_append, "beams": _own_beams, "reorder": _own_reorder}
_plain = {"rotary": _plain_rotary, "append": _plain_append, "beams": _plain_beams, "reorder": _plain_reorder}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "beams":
        rng = random.Random(case["shape"])
        live = sum(rng.random() >= case["ended"] for _ in range(case["batch"] * case["beams"]))
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": live * case["vocab"] * size + case["batch"] * (5 * case["beams"] + 13 * case["n"]),
                "flops": 3.0 * live * case["vocab"]}
    token = 2 * case["hkv"] * case["d"]                     # bytes of one token's keys
    if case["op"] == "rotary":
        rows = case["batch"] * case["tokens"]
        heads, axes = case["hq"] + case["hkv"], 3 if case["sections"] else 1
        return {"bytes": rows * (4 * heads * case["d"] + 4 * axes), "flops": 3.0 * rows * heads * case["part"]}
    lens = _lens(case)
    if case["op"] == "append":
        new, asked = sum(len(x) for x in _accepted(case)), len(lens) * case["tokens"] * case["queries"]
        return {"bytes": 4 * token * new + 4 * case["hq"] * case["d"] * asked,
                "flops": 3.0 * case["part"] * (new * case["hkv"] + asked * case["hq"])}
    grown, beams, page, copied = case["grown"], case["beams"], case["page"], 0
    for n, row in zip(lens, _parents(case)):
        row = [j if p < 0 else p for j, p in enumerate(row)]
        copied += (beams - len(set(row))) * ((n + grown) % page)
    width = max(-(-(n + grown + 1) // page) for n in lens)
    state = 4 * (grown + 1) + (4 * case["hkv"] * width * page if case["weights"] else 0)
    return {"bytes": 4 * token * copied + 2 * len(lens) * beams * (state + 4 * width + 4), "flops": 0}


# ---------------------------------------------------------------- the same in 64 bits
def _exact_rotate(case, x, positions, back=False):
    """x [B, T, H, d] in 64 bits, pair by pair as a product of complex numbers."""
    r = case["part"]
    y = x.double().clone()
    counted = _sections(case) or [r // 2]
    axis = [a for a, n in enumerate(counted) for _ in range(n)]
    for i in range(r // 2):
        f = case["base"] ** (-2.0 * i / r)
        if case["original"]:
            keep = min(1.0, max(0.0, (case["original"] * f / (2 * math.pi) - 1.0) / 3.0))
            f *= keep + (1.0 - keep) / case["factor"]
        else:
            f /= case["factor"]
        at = (positions[axis[i]] if case["sections"] else positions).double() * f
        turn = torch.polar(torch.ones_like(at), -at if back else at)[:, :, None]
        a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + r // 2)
        z = torch.complex(x[..., a].double(), x[..., b].double()) * turn
        y[..., a], y[..., b] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return {n: _exact_rotate(case, s[n], s["positions"], case["back"]) for n in ("q", "k")}
    if case["op"] == "append":
        cache, page, tokens = s["cache"], case["page"], case["tokens"]
        positions = s["positions"]
        if positions is None:
            positions = cache["lens"][:, None] + torch.arange(tokens, device="cuda")
        new = _exact_rotate(case, s["k_new"], positions)
        # The pool in 64 bits, but the means over keys as they are stored.
        k, stored = cache["k"].double(), cache["k"].clone()
        mean = cache["k_mean"].double() if case["means"] else None
        for b, (n, took) in enumerate(zip(_lens(case), _accepted(case))):
            took = torch.tensor(took, device="cuda")
            pos = torch.arange(n, n + len(took), device="cuda")
            ids = cache["table"][b, pos // page].long()
            k[ids, :, pos % page] = new[b, took]
            stored[ids, :, pos % page] = new[b, took].to(stored.dtype)
            if mean is not None:
                for j in range(n // page, -(-(n + len(took)) // page)):
                    held = min(page, n + len(took) - j * page)
                    mean[int(cache["table"][b, j])] = stored[int(cache["table"][b, j])].double()[:, :held].mean(1)
        q = _exact_rotate(case, s["q"], positions) if case["queries"] else None
        return {"k": k, "v": None, "k_mean": mean, "lens": None, "q": q}
    if case["op"] == "beams":
        scores = torch.empty((case["batch"], case["n"]), dtype=torch.float64, device="cuda")
        for b in range(case["batch"]):
            found = []
            for k in range(case["beams"]):
                score = float(s["scores"][b, k])
                if bool(s["finished"][b, k]):
                    found.append(score)
                    continue
                row = s["logits"][b, k].double()
                best = torch.topk(row, min(case["n"], case["vocab"])).values - torch.logsumexp(row, 0)
                found += [score + x for x in best.tolist()]
            found = sorted(found, reverse=True)[:case["n"]]
            scores[b] = torch.tensor(found + [-math.inf] * (case["n"] - len(found)))
        return {"scores": scores, "parent": None, "token": None, "finished": None}
    return None             # copies of what is there
