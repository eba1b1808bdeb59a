"""The decoding-step calls together, as a program uses them: a beam search whose logits come
from the attention over the cache; the same step captured into a graph; calls on
streams of their own."""
import math

import numpy as np
import pytest

from cache_helpers import check_attention, u_of
from oracle import cache as ref_cache
from oracle import decode as ref

pytestmark = pytest.mark.gpu

GROUPS, BEAMS, HQ, HKV, D, PAGE, VOCAB = 2, 3, 4, 2, 64, 16, 500


class Model:
    """Random projections in the place of a model's: of a token, its query, key and value; of its attention, the logits."""

    def __init__(self, dtype, seed=0):
        import torch
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
        self.dtype = dtype
        self.q, self.k, self.v = (rand(VOCAB, h, D).to(dtype) for h in (HQ, HKV, HKV))
        self.out = rand(HQ * D, VOCAB) * 0.3

    def tokens(self, token):
        """q, k, v [B, 1, H, d] of tokens [B] (-1, of a beam without one, as token 0)."""
        t = token.clamp(min=0).long()
        return tuple(x[t][:, None] for x in (self.q, self.k, self.v))

    def logits(self, o):
        return (o.float().reshape(GROUPS, BEAMS, HQ * D) @ self.out).to(self.dtype)


def _start(ev, dtype, prompts, room):
    """A cache whose groups hold their prompts: shared full pages, pages of their own from there."""
    import torch
    rng = np.random.default_rng(4)
    table, at = np.full((GROUPS * BEAMS, -(-(max(prompts) + room) // PAGE)), -1, np.int32), 0
    for g, n in enumerate(prompts):
        f, e = n // PAGE, -(-(n + room) // PAGE)
        table[g * BEAMS:(g + 1) * BEAMS, :f] = at + np.arange(f)
        at += f
        for j in range(BEAMS):
            table[g * BEAMS + j, f:e] = at + np.arange(e - f)
            at += e - f
    pools = [torch.from_numpy(rng.standard_normal((at, HKV, PAGE, D))).to(dtype).cuda() for _ in range(2)]
    for g, n in enumerate(prompts):         # each beam's page in progress holds the prompt's last tokens
        for j in range(1, BEAMS):
            for x in pools:
                x[int(table[g * BEAMS + j, n // PAGE])] = x[int(table[g * BEAMS, n // PAGE])]
    lens = np.repeat(prompts, BEAMS).astype(np.int32)
    return ev.Cache(*pools, torch.from_numpy(table).cuda(), torch.from_numpy(lens).cuda())


def _step(ev, model, rope, cache, logits, scores, ended, text, ws):
    """Beams chosen, their caches and texts taken over, the new tokens appended and attended. ``cache`` becomes the new one."""
    scores, parent, token, ended, _ = ev.evisel_beam_select(logits, scores, finished=ended, eos=7, pad=0, ws=ws)
    cache.table, cache.lens, (text,), _ = ev.evisel_cache_reorder(cache, parent, [text], ws=ws)
    q, k, v = model.tokens(token.reshape(-1))
    cache.lens, q, _ = ev.evisel_cache_append_rotary(cache, rope, k, v, q=q, ws=ws)
    o, lse, _ = ev.evisel_cache_attention(cache, q, ws=ws)
    return dict(scores=scores, parent=parent, token=token, ended=ended, text=text, q=q, o=o, lse=lse, logits=model.logits(o))


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_a_beam_search(cuda_lib, kind):
    """Each step against the oracle: the choice from its logits, what every beam has cached, token by token of its own line
    of parents, and the attention over it."""
    import torch
    ev, dtype = cuda_lib, dict(bf16=torch.bfloat16, fp16=torch.float16)[kind]
    prompts, steps = [37, 16], 20
    model, rope, freqs = Model(dtype), ev.Rotary(D, base=500.0), ref.frequencies(D, 500.0)
    cache, ws = _start(ev, dtype, prompts, steps + 1), ev.Workspace()
    host = lambda x: x.double().cpu().numpy()  # noqa: E731
    lines = []                              # of each sequence: (keys, values) as cached
    for c in range(GROUPS * BEAMS):
        view = dict(k=host(cache.k), v=host(cache.v), table=cache.table.cpu().numpy(), lens=cache.lens.cpu().numpy())
        lines.append([[list(ref_cache.tokens(view, w, c, h)) for h in range(HKV)] for w in "kv"])
    logits = model.logits(torch.randn((GROUPS * BEAMS, 1, HQ, D), device="cuda", generator=torch.Generator("cuda").manual_seed(1)))
    scores = torch.tensor([[0.0, -math.inf, -math.inf]] * GROUPS, device="cuda")         # a prompt's beams are one at first
    ended = torch.zeros((GROUPS, BEAMS), dtype=torch.bool, device="cuda")
    text = torch.full((GROUPS * BEAMS, steps), -1, dtype=torch.int32, device="cuda")
    texts = [[] for _ in range(GROUPS * BEAMS)]
    for i in range(steps):
        before, s = (host(logits), host(scores), ended.cpu().numpy()), None
        s = _step(ev, model, rope, cache, logits, scores, ended, text, ws)
        parent, token = s["parent"].cpu().numpy(), s["token"].cpu().numpy()
        e = 2.0 ** -18 + 2.0 ** -22 + 2.0 ** -23 * (math.log(VOCAB) + 1)
        for g in range(GROUPS):
            want = ref.continuations(before[0][g], before[1][g], before[2][g], 0)
            value = {(k, v): x for x, k, v in want}
            for j in range(BEAMS):
                x = value[int(parent[g, j]), int(token[g, j])]
                assert abs(x - want[j][0]) <= 2 * e and abs(float(s["scores"][g, j]) - x) <= e + 2.0 ** -24 * abs(x)
                assert bool(s["ended"][g, j]) == (token[g, j] == 7 or bool(before[2][g, parent[g, j]]))
        source = (parent + BEAMS * np.arange(GROUPS)[:, None]).reshape(-1)
        lines = [[[list(x) for x in w] for w in lines[p]] for p in source]
        texts = [texts[p] + [int(t)] for p, t in zip(source, token.reshape(-1))]
        text = s["text"]
        text[:, i] = s["token"].reshape(-1)
        assert text[:, :i + 1].tolist() == texts
        # What each beam has cached: its line's tokens as they were, and the new one rotated to its place.
        view = dict(k=host(cache.k), v=host(cache.v), table=cache.table.cpu().numpy(), lens=cache.lens.cpu().numpy())
        q, k, v = (host(x) for x in model.tokens(s["token"].reshape(-1)))
        place = np.repeat(prompts, BEAMS)[:, None] + i
        assert view["lens"].tolist() == (place[:, 0] + 1).tolist()
        k_want, k_size = ref.rotate(k, place, freqs)
        q_want, q_size = ref.rotate(q, place, freqs)
        bound = lambda y, size: (2.0 ** -21 + 2.0 ** -40) * size + u_of(dtype) * np.abs(y) + 2.0 ** -25  # noqa: E731
        assert np.all(np.abs(host(s["q"]) - q_want) <= bound(q_want, q_size))
        for c in range(GROUPS * BEAMS):
            for h in range(HKV):
                got_k, got_v = (ref_cache.tokens(view, w, c, h) for w in "kv")
                assert np.all(np.abs(got_k[-1] - k_want[c, 0, h]) <= bound(k_want[c, 0, h], k_size[c, 0, h]))
                assert np.array_equal(got_k[:-1], np.array(lines[c][0][h])) and np.array_equal(got_v[:-1], np.array(lines[c][1][h]))
                assert np.array_equal(got_v[-1], v[c, 0, h])
                lines[c][0][h].append(got_k[-1])
                lines[c][1][h].append(got_v[-1])
        check_attention(s["o"], s["lse"], ref_cache.attention(view, host(s["q"])), D, dtype, f"step {i}")
        logits, scores, ended = s["logits"], s["scores"], s["ended"]
    assert ev.evisel_status(ws) == 0


def test_a_beam_step_in_a_graph(cuda_lib):
    """The step captured, and replayed on other inputs: the same as the calls one by one, the pages too."""
    import torch
    ev, dtype = cuda_lib, torch.bfloat16
    model, rope, ws = Model(dtype), ev.Rotary(D), ev.Workspace()
    first = _start(ev, dtype, [37, 16], 30)
    held = dict(logits=torch.randn((GROUPS, BEAMS, VOCAB), device="cuda").to(dtype), scores=torch.zeros((GROUPS, BEAMS), device="cuda"),
                ended=torch.zeros((GROUPS, BEAMS), dtype=torch.bool, device="cuda"),
                text=torch.zeros((GROUPS * BEAMS, 9), dtype=torch.int32, device="cuda"))
    k, v, table, lens = (x.clone() for x in (first.k, first.v, first.table, first.lens))
    fresh = lambda: ev.Cache(first.k, first.v, first.table, first.lens)  # noqa: E731
    _step(ev, model, rope, fresh(), ws=ws, **held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        after = fresh()
        got = _step(ev, model, rope, after, ws=ws, **held)
        got.update(table=after.table, lens=after.lens)
    for seed in range(4):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        held["logits"].copy_(torch.randn((GROUPS, BEAMS, VOCAB), device="cuda", generator=gen))
        held["scores"].copy_(-torch.rand((GROUPS, BEAMS), device="cuda", generator=gen))
        held["ended"].copy_(torch.rand((GROUPS, BEAMS), device="cuda", generator=gen) < 0.3)
        held["text"].random_(0, VOCAB, generator=gen)
        first.lens.copy_(torch.tensor([37 + seed] * 3 + [16 + 2 * seed] * 3))
        results = []
        for run in (lambda: graph.replay(), lambda: None):
            first.k.copy_(k), first.v.copy_(v)
            run()
            if results:
                after = fresh()
                got_now = _step(ev, model, rope, after, ws=ws, **held)
                got_now.update(table=after.table, lens=after.lens)
            else:
                got_now = got
            results.append({n: x.clone() for n, x in got_now.items()} | dict(k=first.k.clone(), v=first.v.clone()))
        for n, x in results[0].items():
            assert torch.equal(x, results[1][n]), (seed, n)
    assert ev.evisel_status(ws) == 0 and torch.equal(first.table, table) and lens.shape == first.lens.shape


def test_calls_at_once_on_their_own_streams(cuda_lib):
    """Two selections, rotations and appends at a time, each with its stream and workspace, and a stream given by hand."""
    import torch
    ev, dtype = cuda_lib, torch.bfloat16
    streams = [torch.cuda.Stream() for _ in range(2)]
    rope, jobs = ev.Rotary(D), []
    for i in range(2):
        gen = torch.Generator(device="cuda").manual_seed(i)
        x = torch.randn((8, 4, 30011), device="cuda", generator=gen).to(dtype)
        cache = _start(ev, dtype, [37 + i, 16], 30)
        new = torch.randn((GROUPS * BEAMS, 5, HKV, D), device="cuda", generator=gen).to(dtype)
        jobs.append((x, cache, new))
    torch.cuda.synchronize()

    def run(i, stream, rounds):
        x, cache, new = jobs[i]
        ws, out = ev.Workspace(), []
        for _ in range(rounds):
            a = ev.evisel_beam_select(x, None, 6, ws=ws, stream=stream)[:4]
            b = ev.evisel_rotary(rope, new, new, first=cache.lens, stream=stream)
            c = ev.evisel_cache_append_rotary(cache, rope, new, new, ws=ws, stream=stream)[:1]
            d = ev.evisel_cache_reorder(cache, torch.zeros((GROUPS, BEAMS), dtype=torch.int32, device="cuda"), ws=ws, stream=stream)[:2] \
                if stream is None else ()
            out.append([*a, *b, *c, *d])
        return ws, out

    both = [run(i, s, 10) for i, s in enumerate(streams)]
    torch.cuda.synchronize()
    for i in range(2):
        assert ev.evisel_status(both[i][0]) == 0
        _, (want,) = run(i, None, 1)
        for got in both[i][1]:
            for a, b in zip(got, want):
                assert torch.equal(a, b)


def test_graphs_that_share_a_workspace(cuda_lib):
    """Selections of two sizes captured on one workspace, which grows in between: replayed in any order, each as before."""
    import torch
    ev = cuda_lib
    gen = torch.Generator(device="cuda").manual_seed(3)
    ws, made = ev.Workspace(), []
    for batch, vocab, n in ((1, 5000, 4), (16, 70001, 10)):
        x = torch.randn((batch, 3, vocab), device="cuda", generator=gen).to(torch.bfloat16)
        call = lambda x=x, n=n: ev.evisel_beam_select(x, None, n, ws=ws)[:4]  # noqa: E731
        want = call()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            got = call()
        made.append((graph, got, [a.clone() for a in want]))
    for i in (0, 1, 1, 0, 1, 0):
        graph, got, want = made[i]
        for a in got:
            a.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
    assert ev.evisel_status(ws) == 0
    x = torch.randn((64, 3, 200001), device="cuda", generator=gen).to(torch.bfloat16)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with pytest.raises(ev.EviselError, match="capture"):
        with torch.cuda.graph(graph):
            ev.evisel_beam_select(x, None, 10, ws=ws)           # the workspace would have to grow
    assert torch.equal(ev.evisel_beam_select(x[:1], None, 1, ws=ws)[2][0, 0].cpu(), x[0].float().log_softmax(-1).max(0).values.argmax().int().cpu())
