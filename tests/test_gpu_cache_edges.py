"""Weighing, tree attention and pruning where their kernels take another way: waits that run out,
sequences of fewer slots than new tokens, more caches than are resident at once.
Tolerances: as in test_gpu_cache_ops.py.
"""
import math
import random

import pytest
import torch

from paper_2609_06663_gb300 import ecokv as E
from tests import cache_ref as ref
from tests.test_gpu_cache_ops import places, run_prune, seen_of
from tests.test_gpu_decode import TYPES, U, W, Batch, gen, make_prefix

pytestmark = pytest.mark.gpu
D = 128
PATHS = [("bf16", 0), ("bf16", E.ECOKV_FLAG_FORCE_SIMT), ("f32", 0)]


# ---------------------------------------------------------------- waits that run out
@pytest.mark.parametrize("h_q,h_kv,new,lens,page,rows", [(4, 1, [900, 10], [1000, 10], 64, 5), (28, 4, [61] * 8, [300] * 8, 16, 700)])
def test_weigh_that_gave_up_adds_nothing_left_by_others(h_q, h_kv, new, lens, page, rows):
    """Items that are cut between CTAs, none of which gets a tile: no weight changes, whatever the workspace held."""
    b = Batch(7, h_kv, new, lens, page, "bf16")
    heads, pre = make_prefix(gen(2), [rows] * h_kv, "bf16", False)
    q = torch.randn(b.tokens, h_q, D, generator=gen(1)).bfloat16().cuda()
    lse = torch.full((b.tokens, h_q), 5.0, device="cuda")
    pw, w = torch.rand(h_kv, rows, generator=gen(3)).cuda(), torch.rand(b.k.shape[:3], generator=gen(4)).cuda()
    ws = E.alloc_weigh_workspace(b.tokens, len(new), h_q, h_kv, q.dtype)
    ws[256:].fill_(255)  # (NaN where sums are left)
    got = E.weigh(q, lse, pre, b.cache, pw.clone(), w.clone(), b.starts.cuda(), decay=0.5, ws=ws, timeout_us=2000,
                  flags=E.ECOKV_FLAG_TEST_STALL)
    assert E.ecokv_device_status(ws) == E.ECOKV_ERR_TIMEOUT
    assert torch.equal(got[0], pw) and torch.equal(got[1], w)
    # the next call in this workspace as in a new one
    again = [E.weigh(q, lse, pre, b.cache, pw.clone(), w.clone(), b.starts.cuda(), decay=0.5, ws=x)
             for x in (ws, E.alloc_weigh_workspace(b.tokens, len(new), h_q, h_kv, q.dtype))]
    assert E.ecokv_device_status(ws) == 0
    assert torch.equal(again[0][0], again[1][0]) and torch.equal(again[0][1], again[1][1])
    assert not torch.equal(again[0][1], w)


def test_attend_tree_waits_that_run_out():
    """The injected stall: a status, an untouched context, and the next call as ever."""
    b = Batch(6, 4, [61, 3, 20], [161, 200, 300], 16, "bf16")
    heads, pre = make_prefix(gen(2), [500] * 4, "bf16", False)
    q = torch.randn(b.tokens, 28, D, generator=gen(1)).bfloat16().cuda()
    mask = torch.cat([ref.pack(ref.causal(n), 1) for n in b.new]).cuda()
    ws = E.alloc_attend_workspace(b.tokens, 3, 28, 4, q.dtype)
    good = E.attend_tree(q, pre, b.cache, mask, b.starts.cuda(), ws=ws)
    E.attend_tree(q, pre, b.cache, mask, b.starts.cuda(), ws=ws, flags=E.ECOKV_FLAG_TEST_STALL, timeout_us=20000)
    assert E.ecokv_device_status(ws) == E.ECOKV_ERR_TIMEOUT
    assert torch.equal(E.attend_tree(q, pre, b.cache, mask, b.starts.cuda(), ws=ws), good)
    assert E.ecokv_device_status(ws) == 0
    with pytest.raises(E.EcokvError) as e:
        E.attend_tree(q, pre, b.cache, mask, b.starts.cuda(),
                      flags=E.ECOKV_FLAG_TEST_STALL | E.ECOKV_FLAG_FORCE_SIMT)
    assert e.value.code == E.ECOKV_ERR_UNSUPPORTED


# ---------------------------------------------------------------- fewer slots than new tokens
FEW = [  # h_q, h_kv, new, lengths, page, prefix rows
    (7, 1, [90], [1], 8, 300), (4, 4, [3, 40, 5], [2, 17, 0], 16, 0), (28, 4, [61, 25, 300], [40, 80, 130], 32, 77),
    (8, 8, [200], [131], 16, 5), (64, 1, [35, 2], [33, 1], 64, 0), (12, 4, [513, 4], [500, 4], 128, 20),
]


def with_room(own, new):
    """Every sequence's rows behind rows of zeros, which stand for slots below 0, so that its tokens have one each."""
    return [tuple(torch.cat([torch.zeros(x.shape[0], max(n - x.shape[1], 0), D, dtype=x.dtype), x], 1) for x in kv)
            for kv, n in zip(own, new)]


@pytest.mark.parametrize("dt,flags", PATHS)
@pytest.mark.parametrize("h_q,h_kv,new,lens,page,rows", FEW)
def test_weigh_of_more_tokens_than_slots(h_q, h_kv, new, lens, page, rows, dt, flags):
    """Token i sees the slots up to L - T + i, some none at all; every slot is a new one's."""
    b = Batch(3, h_kv, new, lens, page, dt)
    heads, pre = make_prefix(gen(page), [rows] * h_kv, dt, False)
    q = (2 * torch.randn(b.tokens, h_q, D, generator=gen(9))).to(TYPES[dt])
    lse = 3 + math.log(rows + max(lens)) + torch.rand(b.tokens, h_q, generator=gen(3))
    pw, w = torch.rand(h_kv, rows, generator=gen(4)), torch.rand(b.k.shape[:3], generator=gen(5))
    ws = E.alloc_weigh_workspace(b.tokens, len(new), h_q, h_kv, q.dtype)
    got = E.weigh(q.cuda(), lse.cuda(), pre, b.cache, pw.cuda(), w.cuda(), b.starts.cuda(), decay=0.75, flags=flags, ws=ws)
    assert E.ecokv_device_status(ws) == 0
    own = with_room(b.own, new)
    want_p, want_o, size = ref.weigh(q, lse, [h[0] for h in heads], [k for k, _ in own], new, 1 / math.sqrt(D))
    rel = (140 * size + 40 + b.tokens * (h_q // h_kv) + 10) * U
    add = torch.stack(want_p)
    want = 0.75 * pw.double() + add
    assert bool(((got[0].cpu().double() - want).abs() <= rel * add + 3 * U * want + 1e-37).all())
    left = torch.ones(w.shape, dtype=torch.bool)
    y = got[1].cpu()
    for s, (n, L) in enumerate(zip(new, lens)):
        p, r = places(b, s, range(L))
        left[p, :, r] = False
        was = 0.75 * w[p, :, r].double().t()
        was[:, max(L - n, 0):] = 0.0
        add = want_o[s][:, max(n - L, 0):]
        assert bool(((y[p, :, r].double().t() - was - add).abs() <= rel * add + 3 * U * (was + add) + 1e-37).all()), s
    assert torch.equal(y[left], w[left])


@pytest.mark.parametrize("dt,flags", PATHS)
@pytest.mark.parametrize("kind", ["tree", "random", "all", "causal", "none"])
@pytest.mark.parametrize("h_q,h_kv,new,lens,page,rows", FEW)
def test_attend_tree_of_more_tokens_than_slots(h_q, h_kv, new, lens, page, rows, kind, dt, flags):
    """Slot j is draft j - (L - T)'s; bits of the drafts before them count for nothing."""
    b = Batch(3, h_kv, new, lens, page, dt)
    heads, pre = make_prefix(gen(page), [rows] * h_kv, dt, False)
    rng, words = random.Random(3), -(-max(new) // 64)
    seen = [seen_of(kind, n, rng, gen(7)) for n in new]
    mask = torch.cat([ref.pack(m, words) for m in seen]).cuda()
    for m, n, L in zip(seen, new, lens):
        m[:, :max(n - L, 0)] = False
    q = (2 * torch.randn(b.tokens, h_q, D, generator=gen(9))).to(TYPES[dt])
    lse = torch.full((b.tokens, h_q), 5.0, device="cuda")
    ws = E.alloc_attend_workspace(b.tokens, len(new), h_q, h_kv, q.dtype)
    ws[256:].fill_(255)
    out = E.attend_tree(q.cuda(), pre, b.cache, mask, b.starts.cuda(), lse=lse, ws=ws, flags=flags)
    assert E.ecokv_device_status(ws) == 0
    want, size, wl, mag = ref.attend_masked(q, heads, with_room(b.own, new), seen, 1 / math.sqrt(D))
    d = (140 * mag + 40) * U
    keys = rows + max(lens)
    tol = (2 * d + (keys + 300) * U + W[dt]) * size + W[dt] * want.abs() * (1 + 2 ** -7)
    got = out.cpu().double()
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() - tol).max())
    empty = wl == -math.inf
    assert torch.equal(lse.cpu() == -math.inf, empty) and bool((got[empty] == 0).all())
    assert bool(((lse.cpu().double() - wl)[~empty].abs() <= d + (keys + 300) * U + 4 * U * wl[~empty].abs()).all())


# ---------------------------------------------------------------- many caches pruned
def caches(n, most, seed):
    """Lengths up to `most`, some of no slots, some short."""
    r = random.Random(seed)
    return [r.choice([0, 1, 40, r.randint(41, most), r.randint(41, most), most]) for _ in range(n)]


PRUNE = [  # h_kv, lengths, page, budget, limit, first, recent (152 units: one kernel; 156 and more: two)
    (4, caches(38, 500, 1), 16, 130, 150, 4, 8), (4, caches(39, 500, 2), 16, 130, 150, 4, 8),
    (4, caches(64, 700, 3), 64, 300, 310, 0, 32), (8, caches(20, 300, 4), 8, 64, 64, 64, 0), (1, caches(160, 400, 5), 32, 129, 129, 0, 129),
    (1, caches(153, 200, 6), 128, 1, 40, 0, 0), (3, caches(64, 1300, 7), 256, 999, 1000, 1, 0),
]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("to_page", [0, 8, 64])
@pytest.mark.parametrize("h_kv,lens,page,budget,limit,first,recent", PRUNE)
def test_prune_of_many_caches(h_kv, lens, page, budget, limit, first, recent, to_page, dt):
    b = Batch(sum(lens), h_kv, [0] * len(lens), lens, page, dt, "slot" if budget % 2 else "head")
    w = torch.exp(2 * torch.randn(b.k.shape[:3], generator=gen(8)))
    w[w < 0.4] = 0.0  # many equal ones
    run_prune(b, w, budget, limit, first, recent, to_page, move=None if budget == 64 else "same", alias=budget != 300, dt=dt)


def test_prune_of_many_caches_with_a_bad_page():
    lens = [200] * 50
    for to_other in (False, True):
        b = Batch(3, 4, [0] * 50, lens, 16, "bf16")
        w = torch.rand(b.k.shape[:3], generator=gen(8)).cuda()
        to = Batch(4, 4, [0] * 50, [100] * 50, 32, "bf16").cache if to_other else None
        fresh = E.PagedCache(b.dk.clone(), b.dv.clone(), b.cache.table.clone(), b.cache.lengths)
        good = E.prune(fresh, w, 100, 120, 3, 5, to=to)[1]
        k = (fresh if to is None else to).k_pages.clone()
        if to is not None:
            to.k_pages.zero_()
        b.cache.table[7, 2] = 2 ** 30  # slots 32 .. 47
        ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
        n, idx = E.prune(b.cache, w, 100, 120, 3, 5, to=to, ws=ws)
        assert E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX and n.tolist() == [100] * 50
        others = [s for s in range(50) if s != 7]
        assert torch.equal(idx[others], good[others])
        assert not bool(((idx[7] >= 32) & (idx[7] < 48)).any())
        c = b.cache if to is None else to
        for s in others:
            pages = c.table[s, :4].long().cpu() if to is None else c.table[s, :3].long().cpu()
            assert torch.equal(c.k_pages[pages].nan_to_num(9.0), k[pages].nan_to_num(9.0)), s
