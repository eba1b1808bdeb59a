"""The paged-cache calls against their float64 definitions (oracle/cache.py), at
the sizes, masks and layouts where they can go wrong. Bounds: cache_helpers.
"""
import numpy as np
import pytest

from cache_helpers import check_attention, make_cache, random_tree, tensor, tree_words, u_of
from oracle import cache as ref_cache

pytestmark = pytest.mark.gpu


def _types():
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16}


def _status(ev, ws):
    assert ev.evisel_status(ws) == 0


# --- attention ------------------------------------------------------------------

# lens, T, hq, hkv, d, page, dtype, layout, gain
ATTEND = [
    ([0], 1, 1, 1, 64, 16, "bf16", "hnd", 1.0),                        # nothing cached
    ([1], 1, 7, 1, 128, 64, "bf16", "hnd", 1.0),
    ([63, 64, 65], 1, 4, 2, 64, 64, "bf16", "nhd", 1.0),               # unit edges
    ([127, 128, 129, 0, 300], 1, 28, 4, 128, 128, "bf16", "hnd", 1.0),
    ([1000, 17], 1, 28, 4, 128, 16, "fp16", "nhd", 4.0),               # pages inside units, sharp logits
    ([777], 2, 14, 2, 128, 32, "bf16", "hnd", 4.0),                    # 14 rows
    ([200, 0, 5], 3, 16, 8, 64, 16, "fp16", "hnd", 1.0),
    ([500], 16, 2, 2, 128, 64, "bf16", "hnd", 1.0),                    # 16 rows
    ([500], 17, 1, 1, 64, 64, "bf16", "nhd", 1.0),                     # 17
    ([333, 1], 9, 8, 2, 128, 32, "bf16", "hnd", 4.0),                  # 36 rows
    ([129, 700], 33, 7, 1, 64, 64, "fp16", "hnd", 1.0),                # 231 rows, two mask words
    ([260], 64, 14, 2, 128, 128, "bf16", "hnd", 4.0),                  # 448 rows
    ([640, 64], 37, 4, 1, 128, 16, "bf16", "nhd", 1.0),                # 148 rows
    ([40], 5, 128, 1, 64, 16, "bf16", "hnd", 1.0),                     # a group of 128 heads
]


@pytest.mark.parametrize("lens,t,hq,hkv,d,page,dtype,layout,gain", ATTEND)
def test_attention_of_drafted_trees(cuda_lib, lens, t, hq, hkv, d, page, dtype, layout, gain):
    """Random trees, ragged numbers of drafted tokens, NaN in every slot past a sequence's length."""
    import torch
    rng = np.random.default_rng(len(lens) * 1000 + t)
    ty = _types()[dtype]
    cache, ref = make_cache(rng, lens, hkv, d, page, ty, layout, gain=gain)
    batch = len(lens)
    q, q_ref = tensor(rng, (batch, t, hq, d), ty)
    k, k_ref = tensor(rng, (batch, t, hkv, d), ty, gain)
    v, v_ref = tensor(rng, (batch, t, hkv, d), ty)
    allowed = random_tree(rng, batch, t)
    drafted = rng.integers(0 if t > 1 else 1, t + 1, batch)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, k, v, tree=tree_words(allowed),
                                                 drafted=torch.from_numpy(drafted.astype(np.int32)).cuda())
    _status(cuda_lib, ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref, k_ref, v_ref, allowed, drafted), d, ty)


def _roomy(cache):
    """The same tokens in a table that could hold a million: what the choice of a kernel goes by."""
    import torch
    more = (1 << 20) // cache.page - cache.table.shape[-1]
    return cache.view(torch.nn.functional.pad(cache.table, (0, more), value=-1), cache.lens)


@pytest.mark.parametrize("lens,t,hq,hkv,d,page,dtype,layout,gain", [x for x in ATTEND if x[1] * x[2] // x[3] > 16] + [
    ([300, 0, 129], 12, 4, 2, 64, 16, "fp16", "nhd", 4.0),             # 24 rows of heads of 64
    ([1, 65, 511], 16, 14, 2, 64, 32, "bf16", "hnd", 4.0),             # 112 rows, one slot
    ([2000, 0, 300], 45, 7, 1, 128, 64, "fp16", "hnd", 4.0),           # three slots
])
def test_attention_of_drafted_trees_in_roomy_tables(cuda_lib, lens, t, hq, hkv, d, page, dtype, layout, gain):
    """The same by the kernels that long caches take."""
    import torch
    rng = np.random.default_rng(len(lens) * 2000 + t)
    ty = _types()[dtype]
    cache, ref = make_cache(rng, lens, hkv, d, page, ty, layout, gain=gain)
    batch = len(lens)
    q, q_ref = tensor(rng, (batch, t, hq, d), ty)
    k, k_ref = tensor(rng, (batch, t, hkv, d), ty, gain)
    v, v_ref = tensor(rng, (batch, t, hkv, d), ty)
    allowed = random_tree(rng, batch, t)
    drafted = rng.integers(0, t + 1, batch)
    cache = _roomy(cache)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, k, v, tree=tree_words(allowed),
                                                 drafted=torch.from_numpy(drafted.astype(np.int32)).cuda())
    _status(cuda_lib, ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref, k_ref, v_ref, allowed, drafted), d, ty)
    # heads outside tokens in memory, and one query for all sequences
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q.transpose(1, 2).contiguous().transpose(1, 2), ws=ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref), d, ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q[:1].expand(batch, -1, -1, -1), ws=ws)
    check_attention(o, lse, ref_cache.attention(ref, np.repeat(q_ref[:1], batch, 0)), d, ty)
    _status(cuda_lib, ws)


@pytest.mark.parametrize("per_head", [False, True])
def test_lengths_of_their_own_in_roomy_tables(cuda_lib, per_head):
    """Lengths per KV head, and a view of chosen pages, by the kernel that long caches take."""
    rng = np.random.default_rng(31)
    ty = _types()["bf16"]
    lens = np.array([[0, 130, 77], [513, 1, 256]])
    cache, ref = make_cache(rng, lens if per_head else lens[:, 1], 3, 128, 32, ty, per_head=per_head)
    q, q_ref = tensor(rng, (2, 30, 21, 128), ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(_roomy(cache), q)
    _status(cuda_lib, ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref), 128, ty)


@pytest.mark.parametrize("t", [1, 5, 40])
def test_attention_defaults(cuda_lib, t):
    """A chain without a tree; every token without counts; one tree for all; the cache alone; a scale of its own."""
    rng = np.random.default_rng(t)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, [90, 0, 257], 2, 128, 32, ty)
    q, q_ref = tensor(rng, (3, t, 6, 128), ty)
    k, k_ref = tensor(rng, (3, t, 2, 128), ty)
    v, v_ref = tensor(rng, (3, t, 2, 128), ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, k, v)
    check_attention(o, lse, ref_cache.attention(ref, q_ref, k_ref, v_ref), 128, ty, "chain")
    tree = random_tree(rng, 1, t)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, k, v, tree=tree_words(tree)[0], ws=ws, softmax_scale=0.25)
    check_attention(o, lse, ref_cache.attention(ref, q_ref, k_ref, v_ref, np.repeat(tree, 3, 0), scale=0.25), 128, ty, "one tree")
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, ws=ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref), 128, ty, "cache alone")
    _status(cuda_lib, ws)


def test_attention_rows_without_any_key(cuda_lib):
    """Bits that leave a row nothing, over an empty cache and over one token; and values that no row may see."""
    import torch
    rng = np.random.default_rng(5)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, [0, 1], 1, 64, 16, ty)
    q, q_ref = tensor(rng, (2, 4, 3, 64), ty)
    k, k_ref = tensor(rng, (2, 4, 1, 64), ty)
    v, v_ref = tensor(rng, (2, 4, 1, 64), ty)
    allowed = np.zeros((2, 4, 4), bool)
    allowed[0, 1, 1] = allowed[0, 2, 0] = True
    allowed[1, 3, 1] = True
    want = ref_cache.attention(ref, q_ref, k_ref, v_ref, allowed)
    bad = ~allowed.any(1)                                    # drafted tokens that nobody attends
    k[torch.from_numpy(bad).cuda()] = float("inf")
    v[torch.from_numpy(bad).cuda()] = float("nan")
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, k, v, tree=tree_words(allowed))
    check_attention(o, lse, want, 64, ty)
    assert torch.all(o[0, 0] == 0) and torch.all(o[0, 3] == 0)
    # Token 1's value spoils the rows that attend it and no others.
    v[0, 1] = float("nan")
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, k, v, tree=tree_words(allowed), ws=ws)
    assert torch.isnan(o[0, 1]).all() and not torch.isnan(o[0, [0, 2, 3]]).any() and not torch.isnan(o[1]).any()


def test_attention_of_strided_inputs(cuda_lib):
    """q, k and v as views of one fused projection, outputs given, another stream than the default."""
    import torch
    rng = np.random.default_rng(8)
    ty = _types()["fp16"]
    cache, ref = make_cache(rng, [100, 33], 2, 64, 16, ty)
    x, x_ref = tensor(rng, (2, 6, 8 + 2 + 2, 64), ty)
    o = torch.empty((2, 6, 8, 64), dtype=ty, device="cuda")
    lse = torch.empty((8, 2, 6), device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = cuda_lib.evisel_cache_attention(cache, x[:, :, :8], x[:, :, 8:10], x[:, :, 10:], o=o, lse=lse, stream=stream)
    assert got[0] is o and got[1] is lse
    stream.synchronize()
    check_attention(o, lse, ref_cache.attention(ref, x_ref[:, :, :8], x_ref[:, :, 8:10], x_ref[:, :, 10:]), 64, ty)
    # batch and heads in another order in memory
    q = x[:, :, :8].permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    o2, lse2, _ = cuda_lib.evisel_cache_attention(cache, q, x[:, :, 8:10], x[:, :, 10:])
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("order", ["heads outside tokens", "one query for all sequences", "one token for all"])
def test_many_rows_of_queries_in_other_orders(cuda_lib, order):
    """Queries stored [B, hq, T, d], and ones repeated by a stride of 0: attention and evidence."""
    rng = np.random.default_rng(12)
    ty = _types()["bf16"]
    lens = [300, 129]
    cache, ref = make_cache(rng, lens, 2, 64, 32, ty)
    if order == "heads outside tokens":
        q, _ = tensor(rng, (2, 14, 45, 64), ty)
        q = q.transpose(1, 2)
    elif order == "one query for all sequences":
        q, _ = tensor(rng, (1, 45, 14, 64), ty)
        q = q.expand(2, -1, -1, -1)
    else:
        q, _ = tensor(rng, (2, 1, 14, 64), ty)
        q = q.expand(-1, 45, -1, -1)
    q_ref = q.double().cpu().numpy()
    k, k_ref = tensor(rng, (2, 45, 2, 64), ty)
    v, v_ref = tensor(rng, (2, 45, 2, 64), ty)
    allowed = random_tree(rng, 2, 45)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, k, v, tree=tree_words(allowed))
    check_attention(o, lse, ref_cache.attention(ref, q_ref, k_ref, v_ref, allowed), 64, ty)
    acc, ws = cuda_lib.evisel_cache_evidence(cache, q, lse, ws=ws)
    _status(cuda_lib, ws)
    want = ref_cache.evidence(ref, q_ref, lse.cpu().numpy())
    for b in range(2):
        for h in range(2):                       # A <= 40 here, |LSE| <= 10
            got = acc[b, h, :lens[b]].double().cpu().numpy()
            assert np.all(np.abs(got - want[b][h]) <= (72 * 2.0 ** -24 * 40 + 2.0 ** -18) * want[b][h])


def test_attention_of_pages_in_a_larger_pool(cuda_lib):
    """Keys and values interleaved in one pool [P, 2, hkv, page, d], and heads outside the pages."""
    import torch
    rng = np.random.default_rng(9)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, [150, 70], 2, 128, 32, ty)
    q, q_ref = tensor(rng, (2, 1, 8, 128), ty)
    want = ref_cache.attention(ref, q_ref)
    pool = torch.stack([cache.k, cache.v], 1)
    one = cuda_lib.Cache(pool[:, 0], pool[:, 1], cache.table, cache.lens)
    heads = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (cache.k, cache.v)]
    two = cuda_lib.Cache(*heads, cache.table, cache.lens)
    for c in (one, two):
        o, lse, ws = cuda_lib.evisel_cache_attention(c, q)
        check_attention(o, lse, want, 128, ty)
        _status(cuda_lib, ws)


@pytest.mark.parametrize("t", [1, 12])
def test_attention_of_lengths_per_head(cuda_lib, t):
    rng = np.random.default_rng(10)
    ty = _types()["bf16"]
    lens = [[70, 0, 129], [1, 64, 500]]
    cache, ref = make_cache(rng, lens, 3, 64, 16, ty, per_head=True)
    q, q_ref = tensor(rng, (2, t, 6, 64), ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q)
    _status(cuda_lib, ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref), 64, ty)


def test_attention_is_the_same_twice_and_in_a_graph(cuda_lib):
    """Same bits again, alone, among others and replayed with new lengths."""
    import torch
    rng = np.random.default_rng(11)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, [2000, 900, 3], 4, 128, 64, ty, poison=False)
    q, q_ref = tensor(rng, (3, 2, 28, 128), ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q)
    o2, lse2, _ = cuda_lib.evisel_cache_attention(cache, q, ws=ws)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cuda_lib.evisel_cache_attention(cache, q, ws=ws, o=o2, lse=lse2, stream=torch.cuda.current_stream())
    for lens in ([2000, 900, 3], [1, 555, 0], [1999, 64, 64]):
        cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        ref["lens"] = np.array(lens)
        check_attention(o2, lse2, ref_cache.attention(ref, q_ref), 128, ty, str(lens))


@pytest.mark.parametrize("batch", [40, 300])
@pytest.mark.parametrize("t", [1, 20])
def test_attention_of_many_sequences(cuda_lib, batch, t):
    """More sequences than a warp, and than the warps add up by themselves; most of them short or empty."""
    rng = np.random.default_rng(batch)
    ty = _types()["bf16"]
    lens = rng.choice([0, 0, 1, 5, 64, 65, 200], batch)
    cache, ref = make_cache(rng, lens, 1, 64, 16, ty)
    q, q_ref = tensor(rng, (batch, t, 2, 64), ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q)
    _status(cuda_lib, ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref), 64, ty)
    acc, ws = cuda_lib.evisel_cache_evidence(cache, q, lse, ws=ws)
    want = ref_cache.evidence(ref, q_ref, lse.cpu().numpy())
    for b in range(batch):                       # A <= 40 here
        got = acc[b, 0, :lens[b]].double().cpu().numpy()
        assert np.all(np.abs(got - want[b][0]) <= (72 * 2.0 ** -24 * 40 + 2.0 ** -18) * want[b][0])


@pytest.mark.parametrize("t", [1, 7])
def test_attention_of_any_number_of_sequences(cuda_lib, t):
    """Every way that the lengths are added up: up to a warp's lanes, a few for each lane, the block's."""
    import torch
    rng = np.random.default_rng(t)
    ty = _types()["bf16"]
    lens = rng.choice([0, 1, 30, 64, 65, 130, 200], 330)
    cache, ref = make_cache(rng, lens, 1, 64, 16, ty, poison=False)
    q, q_ref = tensor(rng, (330, t, 2, 64), ty)
    want = ref_cache.attention(ref, q_ref)
    weights = None
    for batch in [*range(1, 40), *range(62, 70), 80, 90, *range(94, 100), *range(126, 132), 160, 161, 200, 255, 256, 257, 300, 330]:
        part = cache.view(cache.table[:batch], cache.lens[:batch])
        o, lse, ws = cuda_lib.evisel_cache_attention(part, q[:batch])
        _status(cuda_lib, ws)
        check_attention(o, lse, [x[:, :batch] if x.ndim == 3 else x[:batch] for x in want], 64, ty, f"{batch} sequences")
        acc, ws = cuda_lib.evisel_cache_evidence(part, q[:batch], lse, ws=ws)
        if weights is None or batch == 330:
            lse_all, _ = cuda_lib.evisel_cache_attention(cache, q)[1:]
            weights = cuda_lib.evisel_cache_evidence(cache, q, lse_all)[0]
        for b in range(batch):
            got, one = acc[b, 0, :lens[b]], weights[b, 0, :lens[b]]
            assert torch.all((got - one).abs() <= 1e-4 * one), f"{batch} sequences, {b}"


@pytest.mark.parametrize("t,d", [(37, 64), (23, 128), (80, 64)])
def test_attention_of_an_odd_number_of_slots(cuda_lib, t, d):
    """Row tiles of two slots and of one, long enough that a CTA goes from one kind to the other in mid-walk."""
    rng = np.random.default_rng(t)
    ty = _types()["bf16"]
    lens = [4300, 3999, 130, 4000, 4100, 3500, 1, 4200]
    cache, ref = make_cache(rng, lens, 4, d, 64, ty, poison=False)
    gq = 7 if d == 64 else 16
    q, q_ref = tensor(rng, (len(lens), t, 4 * gq, d), ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q)
    _status(cuda_lib, ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref), d, ty)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("batch,t,gq,d,tree", [(40, 16, 7, 64, True), (3, 100, 7, 128, True), (1, 333, 2, 64, False),
                                               (9, 40, 4, 128, False), (300, 9, 2, 128, True)])
def test_attention_of_many_drafted_rows(cuda_lib, batch, t, gq, d, tree, dtype):
    """Trees and runs whose joins take rows by tiles: several chunks of drafted keys, odd tails, rows that end early,
    drafted values that are not finite where no row may look."""
    import torch
    rng = np.random.default_rng(batch + t)
    ty = _types()[dtype]
    lens = rng.choice([0, 1, 40, 300], batch)
    cache, ref = make_cache(rng, lens, 2, d, 32, ty)
    q, q_ref = tensor(rng, (batch, t, 2 * gq, d), ty)
    k, k_ref = tensor(rng, (batch, t, 2, d), ty)
    v, v_ref = tensor(rng, (batch, t, 2, d), ty)
    drafted = rng.integers(0, t + 1, batch)
    drafted[0] = t
    allowed = np.zeros((batch, t, t), bool)
    for b in range(batch):
        for i in range(t):
            parent = int(rng.integers(max(0, i - 5), i)) if i and tree else i - 1
            allowed[b, i] = allowed[b, parent] if parent >= 0 and i else False
            allowed[b, i, i] = True
        if tree:
            allowed[b, :, 3] = False             # a token that nobody looks at, itself neither
        allowed[b, :, drafted[b]:] = False
    for b in range(batch):                       # what no row may look at may be anything
        for tok in np.nonzero(~allowed[b, :drafted[b]].any(0))[0]:
            k[b, tok], v[b, tok] = float("inf"), float("nan")
            k_ref[b, tok], v_ref[b, tok] = 0, 0
    o, lse, ws = cuda_lib.evisel_cache_attention(
        cache, q, k, v, tree=tree_words(allowed) if tree else None, drafted=torch.from_numpy(drafted.astype(np.int32)).cuda())
    _status(cuda_lib, ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref, k_ref, v_ref, allowed, drafted), d, ty)


def test_attention_of_the_most_drafted_tokens(cuda_lib):
    """A chain of 1,024 tokens over a short cache: 32 mask words a row."""
    rng = np.random.default_rng(4)
    ty = _types()["fp16"]
    cache, ref = make_cache(rng, [21], 1, 64, 16, ty)
    q, q_ref = tensor(rng, (1, 1024, 1, 64), ty)
    k, k_ref = tensor(rng, (1, 1024, 1, 64), ty)
    v, v_ref = tensor(rng, (1, 1024, 1, 64), ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, k, v)
    check_attention(o, lse, ref_cache.attention(ref, q_ref, k_ref, v_ref), 64, ty)
    with pytest.raises(cuda_lib.EviselError):
        cuda_lib.evisel_cache_attention(cache, q.expand(1, -1, -1, -1).repeat(1, 2, 1, 1))


@pytest.mark.parametrize("t", [1, 24])
def test_attention_without_any_page(cuda_lib, t):
    """A table without columns: only the drafted tokens are there; no drafted token at all; no sequence at all."""
    import torch
    rng = np.random.default_rng(6)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, [0, 0], 2, 64, 16, ty)
    bare = cache.view(cache.table[:, :0], cache.lens)
    q, q_ref = tensor(rng, (2, t, 4, 64), ty)
    k, k_ref = tensor(rng, (2, t, 2, 64), ty)
    v, v_ref = tensor(rng, (2, t, 2, 64), ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(bare, q, k, v)
    _status(cuda_lib, ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref, k_ref, v_ref), 64, ty)
    o, lse, _ = cuda_lib.evisel_cache_attention(cache, q[:, :0], k[:, :0], v[:, :0])
    assert o.shape == (2, 0, 4, 64) and lse.shape == (4, 2, 0)
    none = cache.view(cache.table[:0], cache.lens[:0])
    o, lse, _ = cuda_lib.evisel_cache_attention(none, q[:0])
    assert o.shape == (0, t, 4, 64)
    acc, ws = cuda_lib.evisel_cache_evidence(cache.view(cache.table, cache.lens + 3), q[:, :0], lse.new_zeros((4, 2, 0)))
    assert torch.all(acc == 0)


def test_pages_past_4_gb(cuda_lib):
    """Pages whose byte offsets do not fit 32 bits, in every call."""
    import torch
    rng = np.random.default_rng(7)
    ty = _types()["bf16"]
    small, ref = make_cache(rng, [300, 70], 4, 128, 64, ty, room=64, mean=True, poison=False)
    far, n = 70_000, small.k.shape[0]            # a page is 64 KiB
    pools = []
    for x in (small.k, small.v):
        big = torch.empty((far + n, 4, 64, 128), dtype=ty, device="cuda")
        big[far:] = x
        pools.append(big)
    mean = torch.zeros((far + n, 4, 128), dtype=ty, device="cuda")
    cache = cuda_lib.Cache(*pools, small.table + far * (small.table >= 0).int(), small.lens, mean)
    q, q_ref = tensor(rng, (2, 5, 28, 128), ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q)
    check_attention(o, lse, ref_cache.attention(ref, q_ref), 128, ty)
    o1, lse1, _ = cuda_lib.evisel_cache_attention(cache, q[:, :1], ws=ws)
    check_attention(o1, lse1, ref_cache.attention(ref, q_ref[:, :1]), 128, ty)
    a, _ = cuda_lib.evisel_cache_evidence(cache, q, lse, ws=ws)
    b, _ = cuda_lib.evisel_cache_evidence(small, q, lse, ws=ws)
    assert torch.equal(a, b)
    kv, _ = tensor(rng, (2, 40, 4, 128), ty)
    for c in (cache, small):
        c.lens, _ = cuda_lib.evisel_cache_append(c, kv, kv, ws=ws)
    assert torch.equal(cache.k[far:], small.k) and torch.equal(mean[far:], small.k_mean)
    out = [make_cache(rng, [0, 0], 4, 128, 64, ty, room=64, mean=True, poison=False)[0] for _ in range(2)]
    out[1].table.copy_(out[0].table)
    for c, to in ((cache, out[0]), (small, out[1])):
        to.k.zero_(), to.v.zero_()
        cuda_lib.evisel_cache_evict(c, a, to, 64, ws=ws)
    assert torch.equal(out[0].k, out[1].k) and torch.equal(out[0].v, out[1].v)
    va, pa, _ = cuda_lib.evisel_cache_select(cache, q, 3, ws=ws)
    vb, pb, _ = cuda_lib.evisel_cache_select(small, q, 3, ws=ws)
    assert torch.equal(pa, pb) and torch.equal(va.lens, vb.lens) and torch.equal(va.table, vb.table + far * (vb.table >= 0).int())
    _status(cuda_lib, ws)


# --- evidence -------------------------------------------------------------------

@pytest.mark.parametrize("lens,t,hq,hkv,d,page,dtype,layout", [
    ([0], 1, 1, 1, 64, 16, "bf16", "hnd"),
    ([1, 127, 128, 129], 1, 14, 2, 128, 64, "bf16", "nhd"),
    ([300, 0, 77], 5, 16, 8, 64, 16, "fp16", "hnd"),
    ([1000], 33, 7, 1, 128, 128, "bf16", "hnd"),           # 231 rows
    ([200, 513], 40, 12, 2, 64, 32, "bf16", "hnd"),        # 240 rows
    ([140], 130, 3, 1, 128, 32, "fp16", "nhd"),            # 390 rows
    ([260], 2, 128, 1, 64, 16, "bf16", "hnd"),             # a group of 128 heads
])
def test_evidence(cuda_lib, lens, t, hq, hkv, d, page, dtype, layout):
    """Weights of the attention's own LSE; rows left out by ``use`` and by counts, whose queries are not finite;
    NaN in the slots past each length; written, added to, and entries past a length left alone."""
    import torch
    rng = np.random.default_rng(t * 7 + len(lens))
    ty = _types()[dtype]
    cache, ref = make_cache(rng, lens, hkv, d, page, ty, layout)
    batch = len(lens)
    q, q_ref = tensor(rng, (batch, t, hq, d), ty)
    drafted = rng.integers(1, t + 1, batch)
    n_dev = torch.from_numpy(drafted.astype(np.int32)).cuda()
    use = rng.random((batch, t)) < 0.8
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, drafted=n_dev)
    lse_ref = lse.cpu().numpy()
    want = ref_cache.evidence(ref, q_ref, lse_ref, use, drafted)
    dead = ~use | (np.arange(t) >= drafted[:, None])
    q[torch.from_numpy(dead).cuda()] = float("nan")
    acc = torch.full((batch, hkv, cache.max_tokens + 3), 0.5, device="cuda")
    use_dev = torch.from_numpy(use).cuda()
    logit = np.abs(q_ref).max() * np.sqrt(d) * np.nanmax(np.abs(ref["k"]))     # sum |q k| scale is below this
    rel = (d + 8) * 2.0 ** -24 * logit + 2.0 ** -20 + 2.0 ** -22 * 12
    for add in (False, True):
        got, ws = cuda_lib.evisel_cache_evidence(cache, q, lse, acc=acc, use=use_dev, drafted=n_dev, accumulate=add, ws=ws)
        _status(cuda_lib, ws)
        assert got is acc
        host = acc.double().cpu().numpy()
        for b in range(batch):
            for h in range(hkv):
                n = lens[b]
                err = np.abs(host[b, h, :n] - (2.0 if add else 1.0) * want[b][h])
                assert np.all(err <= rel * 2 * want[b][h] + 1e-30), (b, h, add, err.max())
                assert np.all(host[b, h, n:] == 0.5)


@pytest.mark.parametrize("t", [3, 60])
def test_evidence_of_a_key_that_is_not_finite(cuda_lib, t):
    """An infinite key weighs 0 for rows whose logit is -inf, whatever the rows that do not count hold."""
    import torch
    rng = np.random.default_rng(13)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, [200], 1, 64, 16, ty, poison=False)
    at = ref["table"][0, 2], 0, 5                # token 37
    cache.k[at][0] = float("inf")
    q, _ = tensor(rng, (1, t, 4, 64), ty)
    q[..., 0] = -q[..., 0].abs() - 0.5           # used rows: logit -inf
    use = torch.ones((1, t), dtype=torch.bool, device="cuda")
    use[0, 1] = False
    q[0, 1] = float("nan")
    lse = torch.full((4, 1, t), 5.0, device="cuda")
    acc, ws = cuda_lib.evisel_cache_evidence(cache, q, lse, use=use)
    ref["k"] = cache.k.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = ref_cache.evidence(ref, q.double().cpu().numpy(), lse.cpu().numpy(), use.cpu().numpy())[0][0]
    got = acc[0, 0, :200].double().cpu().numpy()
    assert want[37] == 0 and got[37] == 0
    np.testing.assert_allclose(got, want, rtol=72 * 2.0 ** -24 * 40 + 2.0 ** -18)      # A <= 40
    q[0, 2] = float("nan")                       # a row that counts: every key's sum
    acc, ws = cuda_lib.evisel_cache_evidence(cache, q, lse, use=use, ws=ws)
    assert torch.isnan(acc[0, 0, :200]).all()


def test_evidence_of_all_rows_sums_to_the_cached_share(cuda_lib):
    """Without drafted keys a row's weights sum to 1, so that all of them sum to rows x heads of the group."""
    import torch
    rng = np.random.default_rng(3)
    ty = _types()["bf16"]
    cache, _ = make_cache(rng, [4000, 1234], 4, 128, 64, ty)
    q, _ = tensor(rng, (2, 20, 28, 128), ty, 2.0)
    _, lse, ws = cuda_lib.evisel_cache_attention(cache, q)
    acc, ws = cuda_lib.evisel_cache_evidence(cache, q, lse, ws=ws)
    assert acc.shape == (2, 4, cache.max_tokens)
    # 140 rows' LSEs, each within the bound of cache_helpers at A <= 128 here
    assert torch.all((acc.double().sum(2) - 140).abs() <= 140 * (136 * 2.0 ** -24 * 128 + 2.0 ** -19))


# --- eviction -------------------------------------------------------------------

def _scores(rng, kind, batch, hkv, n):
    x = rng.random((batch, hkv, n)).astype(np.float32)
    if kind == "ties":
        x = np.floor(x * 4).astype(np.float32)
    elif kind == "equal":
        x[:] = 0.25
    elif kind == "signs":
        x = np.where(x < 0.2, -0.0, np.where(x < 0.4, 0.0, (x - 0.7) * 1e-30)).astype(np.float32)
    elif kind == "nan":
        x[x < 0.3] = np.nan
        x[x > 0.9] = np.inf
        x[(x > 0.5) & (x < 0.6)] = -np.inf
    return x


@pytest.mark.parametrize("kind", ["random", "ties", "equal", "signs", "nan"])
@pytest.mark.parametrize("lens,hkv,d,page,out_page,budget,sink,recent,dtype", [
    ([0, 1, 5, 64, 65], 2, 64, 16, 32, 8, 1, 3, "bf16"),
    ([100, 101, 99], 1, 128, 64, 16, 100, 0, 0, "fp16"),          # all, one less, fewer
    ([1500, 3000], 3, 64, 32, 128, 257, 4, 33, "bf16"),
    ([2049], 2, 128, 128, 64, 1, 0, 0, "bf16"),                   # a single token
    ([1025, 40], 2, 128, 16, 16, 40, 10, 30, "bf16"),             # nothing left to choose
])
def test_evict(cuda_lib, kind, lens, hkv, d, page, out_page, budget, sink, recent, dtype):
    import torch
    rng = np.random.default_rng(budget)
    ty = _types()[dtype]
    cache, ref = make_cache(rng, lens, hkv, d, page, ty, poison=False)
    batch = len(lens)
    out, out_ref = make_cache(rng, [0] * batch, hkv, d, out_page, ty, "nhd", room=budget, mean=True, poison=False)
    acc = _scores(rng, kind, batch, hkv, cache.max_tokens + 1)
    before = out.k.clone()
    kept, acc_out, ws = cuda_lib.evisel_cache_evict(cache, torch.from_numpy(acc).cuda(), out, budget, sink=sink, recent=recent)
    _status(cuda_lib, ws)
    kept, acc_out = kept.cpu().numpy(), acc_out.cpu().numpy()
    k, v, mean = (x.double().cpu().numpy() for x in (out.k, out.v, out.k_mean))
    table, touched = out_ref["table"], np.zeros(tuple(out.k.shape[:3]), bool)
    for b in range(batch):
        assert int(out.lens[b]) == min(lens[b], budget)
        for h in range(hkv):
            want = ref_cache.choose(acc[b, h], lens[b], budget, sink, recent)
            n = len(want)
            assert kept[b, h, :n].tolist() == want and np.all(kept[b, h, n:] == -1)
            np.testing.assert_array_equal(acc_out[b, h, :n], acc[b, h, want])
            assert np.all(acc_out[b, h, n:] == 0)
            old_k, old_v = ref_cache.tokens(ref, "k", b, h)[want], ref_cache.tokens(ref, "v", b, h)[want]
            for j in range(-(-n // out_page)):
                m = min(out_page, n - j * out_page)
                at = table[b, j]
                touched[at, h, :m] = True
                np.testing.assert_array_equal(k[at, h, :m], old_k[j * out_page:j * out_page + m])
                np.testing.assert_array_equal(v[at, h, :m], old_v[j * out_page:j * out_page + m])
                part = old_k[j * out_page:j * out_page + m]
                bound = (u_of(ty) + out_page * 2.0 ** -23) * np.abs(part).mean(0)
                assert np.all(np.abs(mean[at, h] - part.mean(0)) <= bound)
    np.testing.assert_array_equal(k[~touched], before.double().cpu().numpy()[~touched])    # nothing else is written


@pytest.mark.parametrize("lens,budget", [([70001], 300), ([70001, 9000], 60000), ([8193, 8192, 4097, 4096], 1000)])
def test_evict_from_long_caches(cuda_lib, lens, budget):
    """More scores than a CTA's threads hold, a cluster's share of them, one CTA's: equal ones among them."""
    import torch
    rng = np.random.default_rng(budget)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, lens, 2, 64, 64, ty, poison=False)
    out, _ = make_cache(rng, [0] * len(lens), 2, 64, 64, ty, room=budget, poison=False)
    acc = _scores(rng, "ties", len(lens), 2, cache.max_tokens) + rng.choice([0, 2.0 ** -20], (len(lens), 2, cache.max_tokens)).astype(np.float32)
    kept, acc_out, ws = cuda_lib.evisel_cache_evict(cache, torch.from_numpy(acc).cuda(), out, budget, sink=3, recent=50)
    _status(cuda_lib, ws)
    for b, n in enumerate(lens):
        for h in range(2):
            want = ref_cache.choose(acc[b, h], n, budget, 3, 50)
            got = kept[b, h].cpu().numpy()
            assert got[:len(want)].tolist() == want and np.all(got[len(want):] == -1)
            np.testing.assert_array_equal(acc_out[b, h, :len(want)].cpu().numpy(), acc[b, h, want])
            slot = torch.arange(len(want), device="cuda")
            src = torch.from_numpy(np.array(want)).cuda()
            take = lambda c, i: c.k[c.table[b, i // 64].long(), h, i % 64]  # noqa: E731
            assert torch.equal(take(out, slot), take(cache, src))


# --- append ---------------------------------------------------------------------

@pytest.mark.parametrize("lens,counts,t,hkv,d,page,dtype,layout,own", [
    ([0, 15, 16, 17], [1, 1, 1, 0], 1, 2, 64, 16, "bf16", "hnd", True),
    ([0, 100, 63], [5, 0, 8], 8, 1, 128, 64, "fp16", "nhd", False),
    ([3], [300], 300, 3, 64, 32, "bf16", "hnd", True),
    ([0, 7], None, 129, 2, 128, 128, "bf16", "nhd", True),
])
def test_append(cuda_lib, lens, counts, t, hkv, d, page, dtype, layout, own):
    """Runs and picked tokens, onto page edges; nothing else of the pool changes; means over old and new tokens."""
    import torch
    rng = np.random.default_rng(t)
    ty = _types()[dtype]
    cache, ref = make_cache(rng, lens, hkv, d, page, ty, layout, room=t, mean=True, poison=False)
    batch = len(lens)
    took = counts or [t] * batch
    x, x_ref = tensor(rng, (batch, t, 2 * hkv, d), ty)       # k and v beside each other
    src = None if own else np.stack([rng.permutation(t) for _ in range(batch)]).astype(np.int32)
    k_before, v_before = cache.k.clone(), cache.v.clone()
    new, ws = cuda_lib.evisel_cache_append(
        cache, x[:, :, :hkv], x[:, :, hkv:], src=None if own else torch.from_numpy(src).cuda(),
        counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"))
    _status(cuda_lib, ws)
    assert new.tolist() == [n + c for n, c in zip(lens, took)] and cache.lens.tolist() == list(lens)
    k, v = ref["k"].copy(), ref["v"].copy()
    for b in range(batch):
        for i in range(took[b]):
            pos, s = lens[b] + i, i if own else src[b, i]
            k[ref["table"][b, pos // page], :, pos % page] = x_ref[b, s, :hkv]
            v[ref["table"][b, pos // page], :, pos % page] = x_ref[b, s, hkv:]
    np.testing.assert_array_equal(cache.k.double().cpu().numpy(), k)
    np.testing.assert_array_equal(cache.v.double().cpu().numpy(), v)
    mean = cache.k_mean.double().cpu().numpy()
    touched = np.zeros(len(k), bool)
    for b in range(batch):
        end = lens[b] + took[b]
        for j in range(lens[b] // page, -(-end // page) if took[b] else 0):
            at, m = ref["table"][b, j], min(page, end - j * page)
            touched[at] = True
            part = k[at, :, :m]
            bound = (u_of(ty) + page * 2.0 ** -23) * np.abs(part).mean(1)
            assert np.all(np.abs(mean[at] - part.mean(1)) <= bound)
    assert np.all(mean[~touched] == 0)


def test_append_then_attend_with_new_lengths(cuda_lib):
    """The lengths that an append returns, assigned to the handle, are the ones the next call reads."""
    rng = np.random.default_rng(1)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, [10, 0], 2, 64, 16, ty, room=8, poison=False)
    k, k_ref = tensor(rng, (2, 8, 2, 64), ty)
    v, v_ref = tensor(rng, (2, 8, 2, 64), ty)
    cache.lens, ws = cuda_lib.evisel_cache_append(cache, k, v)
    q, q_ref = tensor(rng, (2, 1, 4, 64), ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, ws=ws)
    ref.update(k=cache.k.double().cpu().numpy(), v=cache.v.double().cpu().numpy(), lens=np.array([18, 8]))
    check_attention(o, lse, ref_cache.attention(ref, q_ref), 64, ty)


# --- selection ------------------------------------------------------------------

@pytest.mark.parametrize("lens,t,hq,hkv,d,page,n,sink,recent,dtype", [
    ([0, 1, 16, 17, 160], 1, 2, 1, 64, 16, 4, 0, 1, "bf16"),
    ([1000, 300], 1, 28, 4, 128, 16, 9, 2, 3, "bf16"),
    ([2000], 5, 6, 2, 64, 32, 8, 1, 7, "fp16"),               # nothing left to choose
    ([4096, 4033], 12, 14, 2, 128, 64, 64, 1, 1, "bf16"),     # all; one short page
    ([16 * 2100 + 5], 1, 2, 2, 64, 16, 100, 0, 1, "bf16"),    # more pages than a block has threads
])
def test_select(cuda_lib, lens, t, hq, hkv, d, page, n, sink, recent, dtype):
    """Chosen pages against the exact scores (numbers on a grid: no rounding in any order), and the attention over
    them against the attention over those tokens."""
    import torch
    rng = np.random.default_rng(n)
    ty = _types()[dtype]
    cache, ref = make_cache(rng, lens, hkv, d, page, ty, mean=True, poison=False)
    batch = len(lens)
    grid = lambda x: np.clip(np.round(x * 16), -128, 128) / 16  # noqa: E731
    q_ref = grid(rng.standard_normal((batch, t, hq, d)))
    mean = grid(rng.standard_normal((len(ref["k"]), hkv, d)))
    cache.k_mean.copy_(torch.from_numpy(mean))
    q = torch.from_numpy(q_ref).to(ty).cuda()
    drafted = rng.integers(1, t + 1, batch)
    n_dev = torch.from_numpy(drafted.astype(np.int32)).cuda()
    view, pages, ws = cuda_lib.evisel_cache_select(cache, q, n, sink=sink, recent=recent, drafted=n_dev)
    _status(cuda_lib, ws)
    pages = pages.cpu().numpy()
    sel = dict(ref, table=np.zeros((batch, hkv, n), np.int32), lens=np.zeros((batch, hkv), np.int64))
    for b in range(batch):
        count = -(-lens[b] // page)
        for h in range(hkv):
            want = ref_cache.choose(ref_cache.page_scores(ref, mean, q_ref, b, h, drafted), count, n, sink, recent)
            assert pages[b, h, :len(want)].tolist() == want and np.all(pages[b, h, len(want):] == -1)
            sel["table"][b, h, :len(want)] = ref["table"][b, want]
            sel["lens"][b, h] = sum(min(page, lens[b] - j * page) for j in want)
    np.testing.assert_array_equal(view.lens.cpu().numpy(), sel["lens"])
    o, lse, ws = cuda_lib.evisel_cache_attention(view, q, drafted=n_dev, ws=ws)
    _status(cuda_lib, ws)
    check_attention(o, lse, ref_cache.attention(sel, q_ref, drafted=drafted), d, ty)


def test_a_step_in_a_graph(cuda_lib):
    """Append, attention, choice, attention over it, evidence and eviction captured as one graph: the same as the
    calls one by one, also with other lengths and inputs at replay."""
    import torch
    rng = np.random.default_rng(17)
    ty = _types()["bf16"]
    cache, _ = make_cache(rng, [500, 130], 2, 128, 32, ty, room=8, mean=True, poison=False)
    out, _ = make_cache(rng, [0, 0], 2, 128, 32, ty, room=64, mean=True, poison=False)
    q, _ = tensor(rng, (2, 4, 14, 128), ty)
    kv, _ = tensor(rng, (2, 4, 2, 128), ty)
    after = cuda_lib.Cache(cache.k, cache.v, cache.table, cache.lens.clone(), cache.k_mean)

    def step(ws):
        lens, ws = cuda_lib.evisel_cache_append(cache, kv, kv, lens_out=after.lens, ws=ws)
        o, lse, _ = cuda_lib.evisel_cache_attention(after, q, ws=ws)
        view, pages, _ = cuda_lib.evisel_cache_select(after, q, 5, ws=ws)
        o2, lse2, _ = cuda_lib.evisel_cache_attention(view, q, ws=ws)
        acc, _ = cuda_lib.evisel_cache_evidence(after, q, lse, ws=ws)
        kept, acc_out, _ = cuda_lib.evisel_cache_evict(after, acc, out, 64, sink=1, recent=2, ws=ws)
        return [lens, o, lse, pages, o2, lse2, acc, kept, acc_out], ws

    _, ws = step(None)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held, _ = step(ws)
    for lens in ([500, 130], [1, 33], [0, 499]):
        cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        q.copy_(tensor(rng, (2, 4, 14, 128), ty)[0])
        graph.replay()
        got = [x.clone() for x in held]
        want, _ = step(ws)
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), (lens, i)
        # the second sequence has five pages: 499 tokens end beyond them, which the kernels record
        assert cuda_lib.evisel_status(ws) == (0 if lens[1] + 4 <= 5 * 32 else -7), lens


# --- what the kernels catch --------------------------------------------------------

def test_out_of_range_device_values_are_reported(cuda_lib):
    """Lengths, page ids, source indices and counts out of range: no access leaves the buffers, the status says so,
    and the next call is as good as new."""
    import torch
    rng = np.random.default_rng(2)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, [40, 20], 2, 64, 16, ty, room=16, mean=True, poison=False)
    q, q_ref = tensor(rng, (2, 2, 4, 64), ty)
    kv, _ = tensor(rng, (2, 2, 2, 64), ty)
    out, _ = make_cache(rng, [0, 0], 2, 64, 16, ty, room=16, mean=True, poison=False)
    acc = torch.rand((2, 2, cache.max_tokens), device="cuda")
    good_table, good_lens = cache.table.clone(), cache.lens.clone()
    i32 = dict(dtype=torch.int32, device="cuda")

    def calls(c, **kw):
        o, lse, ws = cuda_lib.evisel_cache_attention(c, q)
        yield ws
        yield cuda_lib.evisel_cache_evidence(c, q, lse, acc=acc.clone())[1]
        yield cuda_lib.evisel_cache_evict(c, acc, out, 8)[2]
        yield cuda_lib.evisel_cache_select(c, q, 2)[2]
        yield cuda_lib.evisel_cache_append(c, kv, kv)[1]

    for table, lens in ((good_table + len(ref["k"]), good_lens), (-good_table - 1, good_lens),
                        (good_table, good_lens + 10_000), (good_table, -good_lens)):
        for ws in calls(cache.view(table, lens)):
            assert cuda_lib.evisel_status(ws) == -7
            assert cuda_lib.evisel_status(ws) == 0
    for kw in (dict(src=torch.full((2, 2), 2, **i32)), dict(src=torch.full((2, 2), -1, **i32)),
               dict(counts=torch.tensor([3, 1], **i32)), dict(counts=torch.tensor([-1, 1], **i32))):
        _, ws = cuda_lib.evisel_cache_append(cache, kv, kv, **kw)
        assert cuda_lib.evisel_status(ws) == -7
    full = torch.tensor([cache.max_tokens, 0], **i32)
    new, ws = cuda_lib.evisel_cache_append(cache.view(good_table, full), kv, kv)
    assert new.tolist() == [cache.max_tokens, 2] and cuda_lib.evisel_status(ws) == -7
    # acc shorter than a sequence
    _, lse, ws = cuda_lib.evisel_cache_attention(cache, q, ws=ws)
    short = torch.full((2, 2, 30), -1.0, device="cuda")
    cuda_lib.evisel_cache_evidence(cache, q, lse, acc=short, ws=ws)
    assert cuda_lib.evisel_status(ws) == -7
    cuda_lib.evisel_cache_evict(cache, short, out, 8, ws=ws)
    assert cuda_lib.evisel_status(ws) == -7
    good, ref = make_cache(rng, [40, 20], 2, 64, 16, ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(good, q, ws=ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref), 64, ty)
    _status(cuda_lib, ws)


# --- batches of mostly empty sequences ------------------------------------------------

@pytest.mark.parametrize("roomy,lens,t,hq,hkv,d", [
    (False, [100] + 7 * [0], 1, 28, 4, 128),
    (False, [600] + 31 * [0], 2, 4, 1, 64),
    (False, 15 * [0] + [130], 3, 4, 2, 64),
    (True, [513] + 7 * [0], 40, 14, 2, 128),
    (True, [0, 1100] + 10 * [0], 9, 4, 1, 64),
    (False, [100] + 7 * [0], 64, 28, 4, 128),              # the join by tiles of rows
])
def test_attention_of_mostly_empty_batches(cuda_lib, roomy, lens, t, hq, hkv, d):
    """Fewer units than (sequence, KV head) pairs, on a workspace whose scratch a larger call has filled."""
    rng = np.random.default_rng(t)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, lens, hkv, d, 16, ty, room=8)
    large, _ = make_cache(rng, [900] * len(lens), hkv, d, 64, ty, poison=False)
    if roomy:
        cache, large = _roomy(cache), _roomy(large)
    q, q_ref = tensor(rng, (len(lens), t, hq, d), ty)
    _, _, ws = cuda_lib.evisel_cache_attention(large, q)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, ws=ws)
    _status(cuda_lib, ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref), d, ty)
    k, k_ref = tensor(rng, (len(lens), t, hkv, d), ty)
    v, v_ref = tensor(rng, (len(lens), t, hkv, d), ty)
    o, lse, ws = cuda_lib.evisel_cache_attention(cache, q, k, v, ws=ws)
    _status(cuda_lib, ws)
    check_attention(o, lse, ref_cache.attention(ref, q_ref, k_ref, v_ref), d, ty, "with drafted keys")


# --- what a bad table or length may not write ------------------------------------------

@pytest.mark.parametrize("bad", [-1, -7, "past"])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 32)])
def test_a_bad_page_id_writes_nothing(cuda_lib, bad, d, page):
    """An append onto a page that the table does not have, and an eviction into one: the other sequences' pages (id 0
    among them) and means stay as they were, their own tokens arrive, and the status says so."""
    import torch
    rng = np.random.default_rng(d)
    ty = _types()["bf16"]

    def two(lens):                               # sequence 0 holds pages 0 and 1; sequence 1 page 2 and then a bad one
        k, v = (torch.from_numpy(rng.standard_normal((4, 2, page, d))).to(ty).cuda() for _ in range(2))
        mean = torch.from_numpy(rng.standard_normal((4, 2, d))).to(ty).cuda()
        table = torch.tensor([[0, 1], [2, 4 if bad == "past" else bad]], dtype=torch.int32, device="cuda")
        return cuda_lib.Cache(k, v, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), mean)

    cache = two([page - 2, page])
    before = [x.clone() for x in (cache.k, cache.v, cache.k_mean)]
    k_new, _ = tensor(rng, (2, 5, 2, d), ty)
    v_new, _ = tensor(rng, (2, 5, 2, d), ty)
    _, ws = cuda_lib.evisel_cache_append(cache, k_new, v_new)
    assert cuda_lib.evisel_status(ws) == -7
    for pool, old, x in ((cache.k, before[0], k_new), (cache.v, before[1], v_new)):
        assert torch.equal(pool[0, :, :page - 2], old[0, :, :page - 2]) and torch.equal(pool[0, :, page - 2:], x[0, :2].transpose(0, 1))
        assert torch.equal(pool[1, :, :3], x[0, 2:].transpose(0, 1)) and torch.equal(pool[1, :, 3:], old[1, :, 3:])
        assert torch.equal(pool[2:], old[2:])
    assert torch.equal(cache.k_mean[2:], before[2][2:])
    for i, m in ((0, page), (1, 3)):
        part = cache.k[i, :, :m].double()
        assert torch.all((cache.k_mean[i].double() - part.mean(1)).abs() <= (u_of(ty) + page * 2.0 ** -23) * part.abs().mean(1))

    full, _ = make_cache(rng, [2 * page, 2 * page], 2, d, 16, ty, poison=False)
    out = two([0, 0])
    before = [x.clone() for x in (out.k, out.v, out.k_mean)]
    acc = torch.rand((2, 2, full.max_tokens), device="cuda")
    kept, _, ws = cuda_lib.evisel_cache_evict(full, acc, out, 2 * page - 1, ws=ws)
    assert cuda_lib.evisel_status(ws) == -7
    for pool, old, src in ((out.k, before[0], full.k), (out.v, before[1], full.v)):
        for h in range(2):
            pos = kept[0, h].long()
            want = src[full.table[0, pos // 16].long(), h, pos % 16]
            assert torch.equal(pool[:2, h].reshape(2 * page, d)[:2 * page - 1], want)
        assert torch.equal(pool[1, :, page - 1], old[1, :, page - 1]) and torch.equal(pool[3], old[3])
    assert torch.equal(out.k_mean[3], before[2][3])


def test_a_negative_length_appends_nothing(cuda_lib):
    """A page shared as a prefix by two sequences, one of which has a bad length."""
    import torch
    rng = np.random.default_rng(3)
    ty = _types()["bf16"]
    pools = [torch.from_numpy(rng.standard_normal((3, 1, 16, 64))).to(ty).cuda() for _ in range(2)]
    table = torch.tensor([[0, 1], [0, 2]], dtype=torch.int32, device="cuda")
    cache = cuda_lib.Cache(*pools, table, torch.tensor([16, -16], dtype=torch.int32, device="cuda"))
    before = [x.clone() for x in pools]
    new, _ = tensor(rng, (2, 2, 1, 64), ty)
    _, ws = cuda_lib.evisel_cache_append(cache, new, new)
    assert cuda_lib.evisel_status(ws) == -7
    for pool, old in zip(pools, before):
        assert torch.equal(pool[0], old[0]) and torch.equal(pool[2], old[2])
        assert torch.equal(pool[1, 0, :2], new[0, :, 0]) and torch.equal(pool[1, 0, 2:], old[1, 0, 2:])


# --- a stream of the caller's -----------------------------------------------------------

def test_new_tensors_are_made_on_the_stream_of_the_call(cuda_lib):
    """With ``stream=`` and no outputs given: the results are those of the current stream's calls, however busy that
    one is meanwhile, and the memory of the new tensors is the given stream's."""
    import torch
    rng = np.random.default_rng(21)
    ty = _types()["bf16"]
    cache, _ = make_cache(rng, [700, 300], 2, 64, 16, ty, room=8, mean=True, poison=False)
    out, _ = make_cache(rng, [0, 0], 2, 64, 16, ty, room=64, poison=False)
    q, _ = tensor(rng, (2, 3, 4, 64), ty)
    kv, _ = tensor(rng, (2, 3, 2, 64), ty)
    side, ws = torch.cuda.Stream(), cuda_lib.Workspace()

    def calls(stream):
        o, lse, _ = cuda_lib.evisel_cache_attention(cache, q, kv, kv, ws=ws, stream=stream)
        acc, _ = cuda_lib.evisel_cache_evidence(cache, q, lse, ws=ws, stream=stream)
        kept, acc_out, _ = cuda_lib.evisel_cache_evict(cache, acc, out, 64, sink=1, recent=2, ws=ws, stream=stream)
        view, pages, _ = cuda_lib.evisel_cache_select(cache, q, 5, ws=ws, stream=stream)
        lens, _ = cuda_lib.evisel_cache_append(cache, kv, kv, ws=ws, stream=stream)
        return [o, lse, acc, kept, acc_out, view.table, view.lens, pages, lens]

    want = calls(None)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)               # the current stream is busy for about 0.1 s
    got = calls(side)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(want, got)):
        assert torch.equal(a, b), i
    # Freed while the side stream still runs, none of them may be handed to the current one.
    sizes = [(x.shape, x.dtype, x.data_ptr()) for x in got]
    where = {p for _, _, p in sizes}
    del got
    again = [torch.empty(s, dtype=t, device="cuda") for s, t, _ in sizes]
    assert not where & {x.data_ptr() for x in again}
    assert cuda_lib.evisel_status(ws) == 0


# --- graphs and workspaces that grow -----------------------------------------------------

def test_a_graph_outlives_larger_calls_on_its_workspace(cuda_lib):
    """Graphs of growing batches on one workspace, as a server captures them, replayed after all of them; and within a
    capture a call that needs more scratch is refused, its neighbours are captured."""
    import torch
    rng = np.random.default_rng(23)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, [300, 77, 0, 900, 5, 64], 2, 64, 16, ty, poison=False)
    q, q_ref = tensor(rng, (6, 1, 4, 64), ty)
    ws, graphs = cuda_lib.Workspace(), []
    for batch in (1, 2, 6):
        part = cache.view(cache.table[:batch], cache.lens[:batch])
        o, lse, _ = cuda_lib.evisel_cache_attention(part, q[:batch], ws=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cuda_lib.evisel_cache_attention(part, q[:batch], ws=ws, o=o, lse=lse)
        graphs.append((graph, batch, o, lse))
    long, _ = make_cache(rng, [3000] * 40, 2, 64, 64, ty, poison=False)
    many, _ = tensor(rng, (40, 20, 4, 64), ty)
    held, graph = ws.nbytes, torch.cuda.CUDAGraph()
    o, lse = graphs[-1][2:]
    with torch.cuda.graph(graph):
        with pytest.raises(cuda_lib.EviselError, match="capture"):
            cuda_lib.evisel_cache_attention(long, many, ws=ws)
        with pytest.raises(cuda_lib.EviselError, match="capture"):
            cuda_lib.evisel_cache_attention(cache, q)
        cuda_lib.evisel_cache_attention(cache, q, ws=ws, o=o, lse=lse)
    graphs.append((graph, 6, o, lse))
    assert ws.nbytes == held
    cuda_lib.evisel_cache_attention(long, many, ws=ws)       # outgrows what the graphs use
    assert ws.nbytes > held
    filler = torch.full((64 << 20,), float("nan"), device="cuda")
    for graph, batch, o, lse in graphs + graphs[::-1]:
        o.zero_(), lse.zero_()
        graph.replay()
        _status(cuda_lib, ws)
        want = ref_cache.attention(dict(ref, lens=ref["lens"][:batch]), q_ref[:batch])
        check_attention(o, lse, want, 64, ty, f"{batch} sequences")
    assert torch.isnan(filler).all()


# --- the handle ---------------------------------------------------------------------------

def test_assigned_pages_are_the_ones_that_calls_use(cuda_lib):
    """k, v and k_mean of a handle, and of a view of chosen pages, replaced by assignment; what does not fit is refused
    and changes nothing."""
    import torch
    rng = np.random.default_rng(29)
    ty = _types()["bf16"]
    cache, ref = make_cache(rng, [90, 33], 2, 64, 16, ty, room=8, mean=True, poison=False)
    q, q_ref = tensor(rng, (2, 2, 4, 64), ty)
    old_k, old_v, old_mean = cache.k, cache.v, cache.k_mean          # (alive throughout)
    view, _, ws = cuda_lib.evisel_cache_select(cache, q, 3)
    sel = dict(table=view.table.cpu().numpy(), lens=view.lens.cpu().numpy())
    k, v = (torch.from_numpy(rng.standard_normal(tuple(old_k.shape))).to(ty).cuda() for _ in range(2))
    mean = torch.zeros_like(old_mean)
    for c, where in ((cache, ref), (view, sel)):
        c.k, c.v = k, v
        c.k_mean = mean
        assert c.k is k and c.v is v and c.k_mean is mean
        where.update(k=k.double().cpu().numpy(), v=v.double().cpu().numpy())
        o, lse, _ = cuda_lib.evisel_cache_attention(c, q, ws=ws)
        check_attention(o, lse, ref_cache.attention(where, q_ref), 64, ty)
    before = [x.clone() for x in (old_k, old_v, old_mean)]
    new, _ = tensor(rng, (2, 8, 2, 64), ty)
    cuda_lib.evisel_cache_append(cache, new, new, ws=ws)
    assert all(torch.equal(x, y) for x, y in zip((old_k, old_v, old_mean), before)) and bool((mean != 0).any())
    cache.k_mean = None
    with pytest.raises(cuda_lib.EviselError, match="k_mean"):
        cuda_lib.evisel_cache_select(cache, q, 3, ws=ws)
    for name, bad in (("k", k[1:]), ("v", v.float()), ("k", k.cpu()), ("v", v[..., :32]), ("k_mean", mean[:, :1])):
        with pytest.raises(ValueError):
            setattr(cache, name, bad)
        assert cache.k is k and cache.v is v and cache.k_mean is None
    _status(cuda_lib, ws)


# --- small weights in fp16 ------------------------------------------------------------------

@pytest.mark.parametrize("lens,t,gq,d,roomy,drafted", [
    ([4096, 1000], 1, 4, 64, False, False), ([4096], 1, 7, 128, False, False),       # few rows
    ([4096], 6, 4, 64, True, False),                                                  # 32-row tiles
    ([4096, 300], 40, 4, 64, True, False), ([2048], 20, 7, 128, True, False),         # many rows
    ([0], 128, 4, 64, False, True),                                                   # drafted keys joined by tiles
    ([0], 70, 8, 128, False, True), ([0, 0], 20, 2, 64, False, True),                 # and row by row
])
def test_small_weights_count_in_fp16(cuda_lib, lens, t, gq, d, roomy, drafted):
    """Every sixteenth key has the row's maximum and a value of 0, the others weigh e^-18 = 2^-26 of it and hold all of
    the values. A weight is kept to 2^-32 of the maximum at the least (half an fp16 step of 2^-24, 2^7 above it), so
    that O = sum w v / sum w is off by 2^-32 sum |v| / sum w at most, beside the rounding of each weight and of O to
    11 bits; v is large so that O does not fall among the type's last steps (2^-25 more)."""
    import torch
    rng = np.random.default_rng(t + d)
    ty = torch.float16
    cache, ref = make_cache(rng, lens, 1, d, 16, ty, poison=False)
    batch = len(lens)

    def fill(k, v, axis):                        # k = -18 e_0 but for every sixteenth, v positive but for those
        at = [slice(None)] * k.dim()
        at[axis] = slice(None, None, 16)
        k.zero_(), v.copy_(v.abs() * 10_000 + 20_000).clamp_(max=60_000)
        k[..., 0] = -18.0
        k[tuple(at)] = 0.0
        v[tuple(at)] = 0.0

    fill(cache.k, cache.v, 2)
    ref.update(k=cache.k.double().cpu().numpy(), v=cache.v.double().cpu().numpy())
    q = torch.zeros((batch, t, gq, d), dtype=ty, device="cuda")
    q[..., 0] = 1.0
    k = v = None
    if drafted:
        k, v = (tensor(rng, (batch, t, 1, d), ty)[0] for _ in range(2))
        fill(k, v, 1)
    tree = tree_words(np.ones((batch, t, t), bool)) if drafted else None
    o, lse, ws = cuda_lib.evisel_cache_attention(_roomy(cache) if roomy else cache, q, k, v, tree=tree, softmax_scale=1.0)
    _status(cuda_lib, ws)
    allowed = np.ones((batch, t, t), bool)
    host = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
    o_ref, lse_ref, size, values, _ = ref_cache.attention(ref, host(q), host(k), host(v), allowed, scale=1.0)
    assert o_ref[0].min() > 2.0 ** -11           # the values' share is there to be seen
    total = np.moveaxis(np.exp(lse_ref), 0, 2)[..., None]          # the maximum is e^0
    bound = 2.0 ** -32 * values / total + 2.0 ** -10 * size + 2.0 ** -18 * size + 2.0 ** -25
    err = np.abs(o.double().cpu().numpy() - o_ref)
    assert np.all(err <= bound), f"O off by {err.max():.2e}, {np.max(err / bound):.2f} of the bound"
    e = (d + 8) * 2.0 ** -24 * 18 + 2.0 ** -20
    assert np.all(np.abs(lse.double().cpu().numpy() - lse_ref) <= e + 2.0 ** -22 * np.abs(lse_ref))


# --- caches without a page --------------------------------------------------------------------

def test_every_call_on_a_cache_without_a_page(cuda_lib):
    """No column in the table, as before a first append: evidence of nothing, an eviction that
    keeps nothing, a choice of nothing; and a table with room whose sequences are empty, with weights of no length."""
    import torch
    rng = np.random.default_rng(31)
    ty = _types()["bf16"]
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros((1, 2, 16, 64), dtype=ty, device="cuda")
    bare = cuda_lib.Cache(pool, pool, torch.zeros((3, 0), **i32), torch.zeros(3, **i32),
                          torch.zeros((1, 2, 64), dtype=ty, device="cuda"))
    room, _ = make_cache(rng, [0, 0, 0], 2, 64, 16, ty, room=32, poison=False)
    q, _ = tensor(rng, (3, 2, 4, 64), ty)
    lse = torch.zeros((4, 3, 2), device="cuda")
    for cache in (bare, room):
        none = torch.zeros((3, 2, 0), device="cuda")
        acc, ws = cuda_lib.evisel_cache_evidence(cache, q, lse, acc=none)
        assert acc is none
        out, _ = make_cache(rng, [5, 6, 7], 2, 64, 16, ty, room=8, mean=True, poison=False)
        before = out.k.clone(), out.v.clone(), out.k_mean.clone()
        kept, acc_out, ws = cuda_lib.evisel_cache_evict(cache, none, out, 8, sink=1, recent=2, ws=ws)
        assert torch.all(kept == -1) and torch.all(acc_out == 0) and out.lens.tolist() == [0, 0, 0]
        assert all(torch.equal(x, y) for x, y in zip((out.k, out.v, out.k_mean), before))
        _status(cuda_lib, ws)
    view, pages, ws = cuda_lib.evisel_cache_select(bare, q, 3, ws=ws)
    assert torch.all(pages == -1) and torch.all(view.lens == 0)
    o, lse, ws = cuda_lib.evisel_cache_attention(view, q, ws=ws)
    assert torch.all(o == 0) and torch.all(torch.isneginf(lse))
    _status(cuda_lib, ws)


def test_numbers_past_32_bits_are_refused(cuda_lib):
    """They would reach the library as what is left of them: 2^32 tokens to keep as none."""
    import torch
    rng = np.random.default_rng(37)
    ty = _types()["bf16"]
    cache, _ = make_cache(rng, [40], 1, 64, 16, ty, mean=True, poison=False)
    out, _ = make_cache(rng, [0], 1, 64, 16, ty, room=8, poison=False)
    q, _ = tensor(rng, (1, 1, 2, 64), ty)
    acc = torch.rand((1, 1, cache.max_tokens), device="cuda")
    for name in ("sink", "recent"):
        for n in (1 << 32, -(1 << 32) + 1, 1 << 31):
            with pytest.raises((ValueError, cuda_lib.EviselError)):
                cuda_lib.evisel_cache_evict(cache, acc, out, 8, **{name: n})
            with pytest.raises((ValueError, cuda_lib.EviselError)):
                cuda_lib.evisel_cache_select(cache, q, 2, **{name: n})
    for n in (1 << 31, (1 << 32) + 8):
        with pytest.raises(ValueError, match="32 bits"):
            cuda_lib.evisel_cache_evict(cache, acc, out, n)
        with pytest.raises(ValueError, match="32 bits"):
            cuda_lib.evisel_cache_select(cache, q, n)
