"""Drafted tokens and a cache that shrinks as they are used together: whole steps against their
definitions, in a graph, on other streams, over pages that lie far apart; and the example."""
import importlib.util
import math
import os
import random

import pytest
import torch

from paper_2609_06663_gb300 import ecokv as E
from tests import cache_ref as ref
from tests.test_gpu_cache_ops import ints, places, tree
from tests.test_gpu_decode import TYPES, U, W, Batch, gen, make_prefix
from tests.test_gpu_decode_path import evicted

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
D = 128


class Drafts:
    """A step's drafts: trees, keys, values, queries, and the path that is accepted of each."""

    def __init__(self, seed, new, h_q, h_kv, T):
        rng, g = random.Random(seed), gen(seed)
        self.new, self.trees = new, [tree(rng, n) for n in new]
        self.paths = []
        for t in self.trees:
            at, p = rng.randrange(len(t)) if t else -1, []
            while at >= 0:
                p.append(at)
                at = t[at]
            self.paths.append(p[::-1])
        n = sum(new)
        self.q, self.k, self.v = (torch.randn(n, h, D, generator=g).to(T) for h in (h_q, h_kv, h_kv))
        self.starts = ints([0] + new).cumsum(0).int()
        self.parents = ints([p for t in self.trees for p in t])
        most = max(len(p) for p in self.paths) + 1
        self.accepted = ints([p + [0] * (most - len(p)) for p in self.paths])
        self.counts = ints([len(p) for p in self.paths])
        first = [sum(new[:b]) for b in range(len(new))]
        self.rows = [f + i for f, p in zip(first, self.paths) for i in p]  # the accepted tokens of the call
        self.kept_starts = ints([0] + [len(p) for p in self.paths]).cumsum(0).int()


def room(b, slots):
    """More pages for every sequence, up to so many slots."""
    table = b.table.clone()
    for s, n in enumerate(b.lens):
        for c in range(-(-n // b.page), -(-slots // b.page)):
            table[s, c] = b.free.pop()
    b.cache.table.copy_(table)
    b.table = table


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("adaptive", [False, True])
def test_steps_of_drafts_over_an_evicted_prompt(adaptive, dt):
    """Append, attend, commit, weigh and prune, twice; every output against the definition over the rows that a plain
    list of the cache holds."""
    h_q, h_kv, T = 28, 4, TYPES[dt]
    pre, heads = evicted(adaptive, dt)
    b = Batch(3, h_kv, [0] * 4, [40, 3, 0, 117], 16, dt, spare=60, cols=20)
    room(b, 200)
    w = torch.zeros(b.k.shape[:3], device="cuda")
    pw = torch.zeros(pre.k.shape[:-1], device="cuda")
    weights = [torch.zeros(h_kv, n, dtype=torch.float64) for n in b.lens]
    pweights = [torch.zeros(k.shape[0], dtype=torch.float64) for k, _ in heads]
    slack = 0.0
    for step, new in enumerate([[9, 25, 1, 70], [3, 3, 30, 8]]):
        s = Drafts(step, new, h_q, h_kv, T)
        b.cache.lengths += ints(new)
        q = E.append(b.cache, s.k.cuda(), s.v.cuda(), s.starts, q=s.q.cuda())
        mask = E.tree_mask(s.parents, s.starts)
        lse = torch.empty(q.shape[:2], device="cuda")
        out = E.attend_tree(q, pre, b.cache, mask, s.starts, lse=lse)
        first = 0
        for i, n in enumerate(new):
            b.own[i] = tuple(torch.cat([x, y[first:first + n].transpose(0, 1)], 1) for x, y in zip(b.own[i], (s.k, s.v)))
            first += n
        seen = [ref.reach(t) for t in s.trees]
        want, size, wl, mag = ref.attend_masked(s.q, heads, b.own, seen, 1 / math.sqrt(D))
        d = (140 * mag + 40) * U
        keys = max(len(h[0]) for h in heads) + 400
        tol = (2 * d + (keys + 300) * U + W[dt]) * size + W[dt] * want.abs() * (1 + 2 ** -7)
        assert bool(((out.cpu().double() - want).abs() <= tol).all())
        # the accepted path
        assert E.commit(b.cache, s.accepted, s.counts, s.starts, lengths_out=b.cache.lengths) is b.cache.lengths
        for i, (n, p) in enumerate(zip(new, s.paths)):
            base = b.own[i][0].shape[1] - n
            at = list(range(base)) + [base + x for x in p]
            b.own[i] = tuple(x[:, at] for x in b.own[i])
        assert b.cache.lengths.tolist() == [x.shape[1] for x, _ in b.own]
        # weights
        rows = torch.tensor(s.rows)
        lens = [len(p) for p in s.paths]
        E.weigh(q[rows.cuda()], lse[rows.cuda()], pre, b.cache, pw, w, s.kept_starts, decay=0.5)
        gp, go, span = ref.weigh(s.q[rows], lse.cpu()[rows], [k for k, _ in heads], [k for k, _ in b.own], lens, 1 / math.sqrt(D))
        pweights = [0.5 * x + y for x, y in zip(pweights, gp)]
        weights = [torch.cat([0.5 * x, torch.zeros(h_kv, n, dtype=torch.float64)], 1) + y
                   for x, y, n in zip(weights, go, lens)]
        slack += (140 * span + 40 + len(s.rows) * 7 + 20) * U
        assert bool(((pw.cpu().view(-1).double() - torch.cat(pweights)).abs() <= slack * torch.cat(pweights) + 1e-37).all())
        table, dw = b.cache.table.cpu(), w.cpu()
        for i, x in enumerate(weights):
            p, r = places(b, i, range(x.shape[1]), table=table)
            assert bool(((dw[p, :, r].double().t() - x).abs() <= slack * x + 1e-37).all())
        # pruning by the weights that the device has
        lens, idx = E.prune(b.cache, w, 24, 32, first=2, recent=6, to_weights=w, lengths_out=b.cache.lengths)
        for i in range(4):
            p, r = places(b, i, range(weights[i].shape[1]), table=table)
            at = torch.tensor([ref.prune(dw[p, h, r], 24, 32, 2, 6) for h in range(h_kv)])
            assert torch.equal(idx[i, :, :at.shape[1]].cpu().long(), at) and lens[i] == at.shape[1]
            b.own[i] = tuple(torch.gather(x, 1, at[..., None].expand(-1, -1, D)) for x in b.own[i])
            weights[i] = torch.gather(weights[i], 1, at)
    # what is left, read by the plain attention
    q = torch.randn(4, h_q, D, generator=gen(77)).to(T)
    out = E.attend(q.cuda(), pre, b.cache)
    want, size, _, mag = ref.attend_masked(q, heads, b.own, [torch.ones(1, 1, dtype=torch.bool)] * 4, 1 / math.sqrt(D))
    tol = (2 * (140 * mag + 40) * U + 800 * U + W[dt]) * size + W[dt] * want.abs() * (1 + 2 ** -7)
    assert bool(((out.cpu().double() - want).abs() <= tol).all())


def step_of(s, q, pre, cache, w, pw, bufs, to=None):
    """One step with every output in a buffer of the caller's."""
    mask, out, lse, idx, lens, ws, ws2 = bufs
    E.append(cache, s["k"], s["v"], s["starts"])
    E.tree_mask(s["parents"], s["starts"], mask=mask)
    E.attend_tree(q, pre, cache, mask, s["starts"], out=out, lse=lse, ws=ws)
    E.weigh(q, lse, pre, cache, pw, w, s["starts"], ws=ws2)
    E.commit(cache, s["accepted"], s["counts"], s["starts"], weights=w, lengths_out=lens)
    E.prune(cache, w, 20, 40, 1, 4, to=to, to_weights=None if to is None else w, lengths_out=lens, idx=idx)


def test_a_step_in_a_graph_on_another_stream():
    """Captured once and replayed as the drafts, the tables and the lengths change: the bits of the same calls."""
    h_q, h_kv, T = 8, 2, torch.bfloat16
    heads, pre = make_prefix(gen(2), [333] * h_kv, "bf16", False)
    new = [7, 30, 1]

    def fresh(seed):
        b = Batch(seed, h_kv, [0] * 3, [[60, 30, 100], [3, 90, 0]][seed % 2], 16, "bf16", spare=30, cols=12)
        room(b, 144)
        d = Drafts(seed, new, h_q, h_kv, T)
        d.accepted = torch.nn.functional.pad(d.accepted, (0, 32 - d.accepted.shape[1]))
        b.cache.lengths += ints(new)
        return b, d

    def state(b, d):
        s = dict(k=d.k.cuda(), v=d.v.cuda(), starts=d.starts, parents=d.parents, accepted=d.accepted, counts=d.counts)
        bufs = (torch.zeros(38, 1, dtype=torch.int64, device="cuda"), torch.zeros(38, h_q, D, dtype=T, device="cuda"),
                torch.zeros(38, h_q, device="cuda"), torch.zeros(3, h_kv, 40, dtype=torch.int32, device="cuda"),
                torch.zeros(3, dtype=torch.int32, device="cuda"), E.alloc_attend_workspace(38, 3, h_q, h_kv, T),
                E.alloc_weigh_workspace(38, 3, h_q, h_kv, T))
        return s, d.q.cuda(), torch.rand(100, h_kv, 16, generator=gen(1))[:b.k.shape[0]].cuda().contiguous(), \
            torch.zeros(h_kv, 333, device="cuda"), bufs

    n_pages = max(fresh(i)[0].k.shape[0] for i in range(2))
    b0, d0 = fresh(0)
    k_pages, v_pages = (torch.zeros(n_pages, h_kv, 16, D, dtype=T, device="cuda") for _ in range(2))
    cache = E.PagedCache(k_pages, v_pages, b0.cache.table.clone(), b0.cache.lengths.clone())
    s, q, _, pw, bufs = state(b0, d0)
    w = torch.zeros(n_pages, h_kv, 16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step_of(s, q, pre, cache, w, pw, bufs)
        with torch.cuda.graph(graph, stream=side):
            step_of(s, q, pre, cache, w, pw, bufs)
    torch.cuda.synchronize()
    for i in range(4):
        b, d = fresh(i)
        s1, q1, w1, pw1, bufs1 = state(b, d)
        # the same content in the graph's tensors
        k_pages.zero_(), v_pages.zero_(), w.zero_(), pw.copy_(pw1)
        k_pages[:b.k.shape[0]], v_pages[:b.k.shape[0]], w[:b.k.shape[0]] = b.dk, b.dv, w1
        cache.table.copy_(b.cache.table), cache.lengths.copy_(b.cache.lengths)
        for x in s:
            s[x].copy_(s1[x])
        q.copy_(q1)
        graph.replay()
        torch.cuda.synchronize()
        step_of(s1, q1, pre, b.cache, w1, pw1, bufs1)
        for x, y in zip(bufs[:5] + (pw, w[:b.k.shape[0]], k_pages[:b.k.shape[0]], v_pages[:b.k.shape[0]]),
                        bufs1[:5] + (pw1, w1, b.dk, b.dv)):
            assert torch.equal(x.nan_to_num(55.0), y.nan_to_num(55.0))
        assert E.ecokv_device_status(bufs[5]) == 0 and E.ecokv_device_status(bufs[6]) == 0


@pytest.mark.parametrize("how", ["stream", "handle", "current"])
def test_helpers_run_in_the_order_of_their_stream(how):
    """With nothing given but the inputs, while torch's current stream is busy with readers of memory it has given back."""
    h_q, h_kv, T = 8, 2, torch.bfloat16
    new = [7, 30, 1]
    d = Drafts(1, new, h_q, h_kv, T)
    heads, pre = make_prefix(gen(2), [333] * h_kv, "bf16", False)

    def calls(**kw):
        b = Batch(5, h_kv, new, [60, 30, 100], 16, "bf16")
        w = torch.rand(b.k.shape[:3], generator=gen(1)).cuda()
        lse = torch.full((38, h_q), 6.0, device="cuda")
        q, pw = d.q.cuda(), torch.zeros(h_kv, 333, device="cuda")
        torch.cuda.synchronize()
        mask = E.tree_mask(d.parents, d.starts, **kw)
        out = E.attend_tree(q, pre, b.cache, mask, d.starts, **kw)
        E.weigh(q, lse, pre, b.cache, pw, w, d.starts, **kw)
        lens = E.commit(b.cache, d.accepted, d.counts, d.starts, weights=w, **kw)
        lens2, idx = E.prune(b.cache, w, 20, 25, 1, 4, **kw)
        return mask, out, pw, w, lens, lens2, idx, b.dk, b.dv

    want = [x.clone() for x in calls()]
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        for _ in range(20):
            big @ big
        old = [torch.ones_like(x) for x in want]
        kept = [x.clone() for x in old]
        del old
        if how == "current":
            with torch.cuda.stream(side):
                got = calls()
        else:
            got = calls(stream=side if how == "stream" else side.cuda_stream)
        side.synchronize()
        assert all(torch.equal(x.nan_to_num(55.0), y.nan_to_num(55.0)) for x, y in zip(got, want))
        torch.cuda.synchronize()
        assert all(bool((x == 1).all()) for x in kept)


def test_two_calls_at_once():
    """Two streams, a workspace each: nothing of one call is another's."""
    h_q, h_kv, T = 28, 4, torch.bfloat16
    jobs = []
    for i in range(2):
        b = Batch(i, h_kv, [61, 20, 3], [161, 420, 33], 32, "bf16")
        heads, pre = make_prefix(gen(i), [2000] * h_kv, "bf16", False)
        q = torch.randn(84, h_q, D, generator=gen(i)).to(T).cuda()
        lse = torch.full((84, h_q), 8.0, device="cuda")
        jobs.append((b, pre, q, lse, E.alloc_weigh_workspace(84, 3, h_q, h_kv, T), torch.cuda.Stream()))

    def run(i, stream=None):
        b, pre, q, lse, ws, _ = jobs[i]
        w, pw = torch.zeros(b.k.shape[:3], device="cuda"), torch.zeros(h_kv, 2000, device="cuda")
        torch.cuda.synchronize() if stream is None else stream.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            E.weigh(q, lse, pre, b.cache, pw, w, b.starts.cuda() if stream is None else starts[i], ws=ws, stream=stream)
        return pw, w

    starts = [j[0].starts.cuda() for j in jobs]
    want = [run(0), run(1)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [run(i, jobs[i][5]) for i in range(2)]
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_pages_that_lie_far_apart(dt):
    """Offsets past 2^32 bytes and 2^31 elements."""
    T, h_kv, page, far = TYPES[dt], 2, 16, 2 ** 28
    lens, new = [70, 33], [9, 20]
    b = Batch(2, h_kv, new, lens, page, dt)
    n = b.k.shape[0]
    assert far * (n - 1) > 2 ** 31
    flat = [torch.empty(far * (n - 1) + h_kv * page * D, dtype=T, device="cuda") for _ in range(2)]
    k, v = (x.as_strided((n, h_kv, page, D), (far, page * D, D, 1)) for x in flat)
    wide = torch.empty(far * (n - 1) + h_kv * page, device="cuda")
    w = wide.as_strided((n, h_kv, page), (far, page, 1))
    k.copy_(b.dk), v.copy_(b.dv)
    cache = E.PagedCache(k, v, b.cache.table, b.cache.lengths)
    near = torch.rand(n, h_kv, page, generator=gen(1)).cuda()
    w.copy_(near)
    q = torch.randn(29, 4, D, generator=gen(3)).to(T).cuda()
    lse = torch.full((29, 4), 4.0, device="cuda")
    mask = torch.cat([ref.pack(ref.reach(tree(random.Random(i), x)), 1) for i, x in enumerate(new)]).cuda()
    starts = b.starts.cuda()
    assert torch.equal(E.attend_tree(q, None, cache, mask, starts), E.attend_tree(q, None, b.cache, mask, starts))
    E.weigh(q, lse, None, cache, None, w, starts), E.weigh(q, lse, None, b.cache, None, near, starts)
    acc, counts = ints([[1, 3, 8], [0, 5, 19]]), ints([3, 3])
    E.commit(cache, acc, counts, starts, weights=w), E.commit(b.cache, acc, counts, starts, weights=near)
    i1, i2 = (E.prune(c, x, 20, 30, 1, 4, to_weights=x)[1] for c, x in ((cache, w), (b.cache, near)))
    assert torch.equal(i1, i2) and torch.equal(w.nan_to_num(9.0), near.nan_to_num(9.0))
    assert torch.equal(k.nan_to_num(9.0), b.dk.nan_to_num(9.0)) and torch.equal(v.nan_to_num(9.0), b.dv.nan_to_num(9.0))


def test_a_prefix_is_evicted_again_by_its_weights():
    """prefix_weights are what the library's selection and compaction take as scores."""
    h_kv, n, T = 2, 400, torch.bfloat16
    heads, pre = make_prefix(gen(2), [n] * h_kv, "bf16", False)
    q = (2 * torch.randn(50, 8, D, generator=gen(3))).to(T).cuda()
    lse = torch.empty(50, 8, device="cuda")
    E.attend(q, pre, None, lse=lse)
    pw, _ = E.weigh(q, lse, pre, None, torch.zeros(h_kv, n, device="cuda"))
    p = E.make_params(n_layers=1, h_kv=h_kv, h_q=8, n=n, window=4, budget=100)
    idx = E.select(p, pw[None, :, :n - 4].contiguous())
    k, v = E.compact(p, pre.k[None].contiguous(), pre.v[None].contiguous(), idx)
    for h in range(h_kv):
        at = ref.prune(pw[h].cpu(), 100, 100, 0, 4)
        assert idx[0, h].tolist() == at and torch.equal(k[0, h], pre.k[h, at]) and torch.equal(v[0, h], pre.v[h, at])


def test_example_of_draft_trees():
    spec = importlib.util.spec_from_file_location("draft_trees", os.path.join(ROOT, "examples", "draft_trees.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    lengths, accepted = ex.run(tokens=700, batch=5, steps=6, limit=48, budget=32, log=lambda *_: None)
    assert len(accepted) == 6 and all(0 < int(x) <= 48 for x in lengths)
