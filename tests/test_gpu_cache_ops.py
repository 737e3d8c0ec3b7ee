"""Drafted tokens (tree_mask, attend_tree, commit) and a cache that shrinks (weigh, prune) against their definitions in 64 bits.

Tolerances.  u = 2^-24, w = 2^-8 (bf16's rounding) or 0 for fp32.

Attention: as in test_gpu_decode.py.

Weights: a score is a sum of 128 products, off by at most 128 u of sum |q||k| scale; the
scale, the reference (lse log2 e, of the float32 lse that the definition takes too) and their
sum add a few u of it and of |lse|, the exponential 2^-21: with size = sum |q||k| scale +
|lse| an addend is off by (140 size + 40) u relative.  Addends are not negative: a sum of n of
them adds (n + 10) u of it, decay * A and the last addition 2 u of the result.

What is moved, indices, masks and lengths: exact.
"""
import math
import random

import pytest
import torch

from paper_2609_06663_gb300 import ecokv as E
from tests import cache_ref as ref
from tests.test_gpu_decode import TYPES, U, W, Batch, gen, make_prefix

pytestmark = pytest.mark.gpu
D = 128
SIMT = E.ECOKV_FLAG_FORCE_SIMT


def tree(rng, n, kind="mixed"):
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "flat":
        return [-1] * n
    return [-1 if i == 0 or rng.random() < 0.1 else rng.randint(max(0, i - 5), i - 1) if rng.random() < 0.5
            else rng.randint(0, i - 1) for i in range(n)]


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


# ---------------------------------------------------------------- tree_mask
@pytest.mark.parametrize("kind", ["mixed", "chain", "flat"])
@pytest.mark.parametrize("new,words", [([1], 1), ([25], 1), ([64, 0, 65, 1, 63], 2), ([200, 3, 129], 4), ([512], 9),
                                       ([4096, 1], 64), ([1] * 70, 1), ([0, 0, 7], 1), ([33] * 40, 1)])
def test_tree_mask(new, words, kind):
    rng = random.Random(str((new, words)))
    trees = [tree(rng, n, kind) for n in new]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    pad = 3  # tokens of no sequence
    parents = ints([p for t in trees for p in t] + [2 ** 30] * pad)
    mask = torch.full((starts[-1] + pad, words), 77, dtype=torch.int64, device="cuda")
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    assert E.tree_mask(parents, ints(starts), mask=mask, ws=ws) is mask
    want = torch.cat([ref.pack(ref.reach(t), words) for t in trees] + [torch.full((pad, words), 77)])
    assert torch.equal(mask.cpu(), want) and E.ecokv_device_status(ws) == 0


def test_tree_mask_of_single_drafts_and_by_default():
    assert torch.equal(E.tree_mask(ints([-1] * 5)).cpu(), torch.ones(5, 1, dtype=torch.int64))
    got = E.tree_mask(ints(list(range(-1, 69))), ints([0, 70]))
    assert got.shape == (70, 2) and torch.equal(got.cpu(), ref.pack(ref.causal(70), 2))
    assert E.tree_mask(ints([]).int(), ints([0, 0])).shape == (0, 1)


def test_tree_mask_bad_parents():
    for parents, starts, words, want in (
            ([-1, 1, 0, 1], [0, 4], 1, [-1, -1, 0, 1]), ([-2, 0, 5, 2], [0, 4], 1, [-1, 0, -1, 2]),
            ([-1, 0, 2 ** 31 - 1], [0, 3], 1, [-1, 0, -1]), ([-1, -2 ** 31], [0, 2], 1, [-1, -1])):
        ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
        got = E.tree_mask(ints(parents), ints(starts), words=words, ws=ws)
        assert torch.equal(got.cpu(), ref.pack(ref.reach(want), words))
        assert E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX
    # more drafts than the mask has bits; starts out of range
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    got = E.tree_mask(ints([-1] + [0] * 69), ints([0, 70]), words=1, ws=ws).cpu()
    assert torch.equal(got[:64], ref.pack(ref.reach([-1] + [0] * 63), 1)) and bool((got[64:] == 0).all())
    assert E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX
    for starts in ([-3, 2, 3], [0, 2, 9], [0, 3, 1]):
        ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
        E.tree_mask(ints([-1, 0, -1]), ints(starts), ws=ws)
        assert E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX


# ---------------------------------------------------------------- attend_tree
def seen_of(kind, n, rng, g):
    if kind == "tree":
        return ref.reach(tree(rng, n))
    if kind == "causal":
        return ref.causal(n)
    if kind == "none":
        return torch.zeros(n, n, dtype=torch.bool)
    if kind == "all":
        return torch.ones(n, n, dtype=torch.bool)
    return torch.rand(n, n, generator=g) < 0.3


TREE = [  # h_q, h_kv, new, lengths, page, prefix rows (a list: uneven), order
    (4, 4, [1], [1], 16, 0, "head"),
    (4, 2, [1, 1], [5, 130], 8, 1, "head"),
    (28, 4, [25], [65], 16, 205, "head"),
    (28, 4, [7, 25, 0, 61], [7, 300, 12, 189], 32, 385, "slot"),
    (8, 8, [200, 3, 31], [456, 3, 128], 16, 128, "head"),              # drafts over several tiles of keys
    (32, 8, [33, 64, 65], [160, 191, 66], 64, [0, 300, 1, 128, 77, 5, 0, 9], "head"),
    (8, 1, [150], [300], 512, 40, "slot"),                             # many token groups of one sequence
    (64, 1, [1, 2, 35], [9, 20, 500], 256, 64, "head"),                # the largest group
    (6, 2, [2, 2, 40, 2], [2, 2, 40, 30], 16, 0, "head"),              # nothing before the drafts
    (7, 1, [513, 4], [700, 4], 128, 20, "head"),
    (40, 40, [3] * 3, [40, 50, 600], 16, [i % 7 * 40 for i in range(40)], "head"),
]


@pytest.mark.parametrize("dt,flags", [("bf16", 0), ("bf16", SIMT), ("f32", 0)])
@pytest.mark.parametrize("kind", ["tree", "random", "none", "all", "causal"])
@pytest.mark.parametrize("h_q,h_kv,new,lens,page,prefix,order", TREE)
def test_attend_tree(h_q, h_kv, new, lens, page, prefix, order, kind, dt, flags):
    T = TYPES[dt]
    uneven = isinstance(prefix, list)
    b = Batch(sum(lens) + page, h_kv, new, lens, page, dt, order)
    heads, pre = make_prefix(gen(page), prefix if uneven else [prefix] * h_kv, dt, uneven)
    check_tree(b, heads, pre, h_q, kind, dt, flags)


def check_tree(b, heads, pre, h_q, kind, dt, flags=0, extra=1, scale=0.0):
    T, g = TYPES[dt], gen(7)
    rng = random.Random(3)
    seen = [seen_of(kind, n, rng, g) for n in b.new]
    words = -(-max(b.new) // 64) + extra
    mask = torch.cat([ref.pack(m, words) for m in seen])
    for t, n in zip(range(b.tokens), [n for n in b.new for _ in range(n)]):  # bits past the sequence's are not read
        if n < 64 * words:
            w, j = n // 64, n % 64
            mask[t, w] |= -(1 << j)
            mask[t, w + 1:] = -1
    q = (2 * torch.randn(b.tokens, h_q, D, generator=gen(9))).to(T)
    one = all(n == 1 for n in b.new)
    lse = torch.full((b.tokens, h_q), 5.0, device="cuda")
    ws = E.alloc_attend_workspace(b.tokens, len(b.new), h_q, b.h_kv, T)
    ws[256:].fill_(255)  # what a call does not write it must not read
    call = lambda **kw: E.attend_tree(q.cuda(), pre, b.cache, mask.cuda(), None if one else b.starts.cuda(),  # noqa: E731
                                      ws=ws, flags=flags, scale=scale, **kw)
    out = call(lse=lse)
    assert E.ecokv_device_status(ws) == 0
    want, size, wl, mag = ref.attend_masked(q, heads, b.own, seen, scale or 1 / math.sqrt(D))
    d = (140 * mag + 40) * U
    keys = max([len(h[0]) for h in heads] + [0]) + max(b.lens)
    tol = (2 * d + (keys + 300) * U + W[dt]) * size + W[dt] * want.abs() * (1 + 2 ** -7)
    got = out.cpu().double()
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() - tol).max())
    empty = wl == -math.inf
    assert torch.equal(lse.cpu() == -math.inf, empty) and bool((got[empty] == 0).all())
    assert bool(((lse.cpu().double() - wl)[~empty].abs() <= d + (keys + 300) * U + 4 * U * wl[~empty].abs()).all())
    assert torch.equal(call(), out)  # the same bits every time
    return out


def test_attend_tree_refuses_what_does_not_fit():
    b = Batch(1, 2, [1] * 3, [4, 5, 6], 8, "bf16")
    q = torch.zeros(3, 4, D, dtype=torch.bfloat16, device="cuda")
    m = torch.ones(3, 1, dtype=torch.int64, device="cuda")
    for mask in (m.int(), m[:2], m[:, 0], m.cpu(), torch.ones(3, 2, dtype=torch.int64, device="cuda")[:, :1]):
        with pytest.raises(ValueError):
            E.attend_tree(q, None, b.cache, mask)
    with pytest.raises(ValueError):
        E.attend_tree(q, None, None, m)
    with pytest.raises(E.EcokvError) as e:
        E.attend_tree(q, None, b.cache, torch.ones(3, 65, dtype=torch.int64, device="cuda"))
    assert e.value.code == E.ECOKV_ERR_UNSUPPORTED


def test_attend_tree_bad_pages():
    b = Batch(2, 2, [3, 2, 4], [40, 60, 33], 16, "bf16")
    q = torch.randn(9, 4, D, generator=gen(1)).bfloat16().cuda()
    mask = torch.cat([ref.pack(ref.causal(n), 1) for n in b.new]).cuda()
    ws = E.alloc_attend_workspace(9, 3, 4, 2, torch.bfloat16)
    good = E.attend_tree(q, None, b.cache, mask, b.starts.cuda(), ws=ws)
    for bad in (2 ** 30, -5):
        ws = E.alloc_attend_workspace(9, 3, 4, 2, torch.bfloat16)
        table = b.cache.table.clone()
        table[1, 1] = bad
        out = E.attend_tree(q, None, E.PagedCache(b.dk, b.dv, table, b.cache.lengths), mask, b.starts.cuda(), ws=ws)
        assert E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX
        assert torch.equal(out[:3], good[:3]) and torch.equal(out[5:], good[5:])


# ---------------------------------------------------------------- commit
def weights_like(b, seed):
    w = torch.rand(b.k.shape[:3], generator=gen(seed)) * 3
    return w


def places(b, seq, slots, page=None, table=None):
    t, n = (b.table if table is None else table), page or b.page
    s = torch.as_tensor(slots, dtype=torch.long)
    return t[seq, s // n].long(), s % n


COMMIT = [  # h_kv, new, kept before, page, most
    (2, [1], [0], 8, 1), (4, [25, 3, 1], [40, 0, 15], 16, 25), (8, [61] * 5, [7, 100, 3, 64, 250], 32, 30),
    (1, [700, 0, 300], [5, 9, 1000], 128, 700), (3, [9] * 40, list(range(40)), 16, 9), (2, [64, 200], [63, 4000], 4096, 200),
]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("h_kv,new,kept,page,most", COMMIT)
def test_commit(h_kv, new, kept, page, most, own, dt):
    rng = random.Random(str(new))
    lens = [n + k for n, k in zip(new, kept)]
    b = Batch(11, h_kv, new, lens, page, dt, "slot" if own else "head")
    w = weights_like(b, 4) if own else None
    lists = [sorted(rng.sample(range(n), min(n, rng.choice([0, 1, n // 2, n, most])))) for n in new]
    acc = torch.tensor([x[:most] + [-7] * (most - len(x)) for x in lists], dtype=torch.int32)
    counts = [min(len(x), most) for x in lists]
    k, v, ww = b.k.clone(), b.v.clone(), None if w is None else w.clone()
    for s, (n, x, c) in enumerate(zip(new, lists, counts)):
        base = lens[s] - n
        at, to = places(b, s, [base + i for i in x[:c]]), places(b, s, range(base, base + c))
        for y, z in ((k, b.k), (v, b.v), (ww, w)):
            if y is not None:
                y[to[0], :, to[1]] = z[at[0], :, at[1]]
    dw = None if w is None else w.cuda()
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    out = E.commit(b.cache, acc.cuda(), ints(counts), None if all(n == 1 for n in new) else b.starts.cuda(), weights=dw,
                   lengths_out=b.cache.lengths if own else None, ws=ws)
    assert (out is b.cache.lengths) == own and E.ecokv_device_status(ws) == 0
    assert out.tolist() == [k_ + c for k_, c in zip(kept, counts)]
    for got, want in ((b.dk, k), (b.dv, v), (dw, ww)):
        if got is not None:
            assert torch.equal(got.cpu().nan_to_num(123.0), want.nan_to_num(123.0))


def test_commit_of_bad_lists():
    for acc, counts in (([1, 0, 2], 3), ([0, 0, 2], 3), ([0, 1, 5], 3), ([-1, 1, 2], 2), ([0, 1, 2], 4), ([0, 1, 2], -1)):
        b = Batch(1, 2, [5, 5], [20, 30], 8, "bf16")
        ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
        out = E.commit(b.cache, ints([acc, [1, 3, 4]]), ints([counts, 3]), b.starts.cuda(), ws=ws)
        assert out.tolist() == [15, 28] and E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX
        at = places(b, 0, range(20))
        assert torch.equal(b.dk.cpu()[at[0], :, at[1]], b.k[at[0], :, at[1]])
        at, to = places(b, 1, [26, 28, 29]), places(b, 1, [25, 26, 27])
        assert torch.equal(b.dv.cpu()[to[0], :, to[1]], b.v[at[0], :, at[1]])
    b = Batch(1, 2, [5, 5], [20, 30], 8, "bf16")
    b.cache.table[0, 2] = 2 ** 30  # the page of slots 16 .. 19
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    out = E.commit(b.cache, ints([[1, 2], [0, 2]]), ints([2, 2]), b.starts.cuda(), ws=ws)
    assert out.tolist() == [17, 27] and E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX
    with pytest.raises(ValueError):
        E.commit(b.cache, ints([1, 2]), ints([2, 2]), b.starts.cuda())
    with pytest.raises(ValueError):
        E.commit(b.cache, ints([[1, 2]] * 2), ints([2, 2]), b.starts.cuda(), weights=torch.zeros(3, device="cuda"))
    with pytest.raises(E.EcokvError):
        both = torch.zeros(3, dtype=torch.int32, device="cuda")
        c = E.PagedCache(b.dk, b.dv, b.cache.table, both[:2])
        E.commit(c, ints([[1, 2]] * 2), ints([2, 2]), b.starts.cuda(), lengths_out=both[1:])


# ---------------------------------------------------------------- weigh
WEIGH = [  # h_q, h_kv, new, lengths, page, prefix rows (a list: uneven), order
    (4, 4, [1], [1], 16, 0, "head"),
    (4, 2, [1, 1], [5, 130], 8, 1, "head"),
    (28, 4, [1] * 5, [1, 16, 17, 128, 529], 16, 300, "slot"),
    (28, 4, [1] * 40, [1 + 17 * i for i in range(40)], 32, 129, "head"),
    (8, 8, [3, 0, 5, 1], [3, 40, 200, 640], 16, 128, "head"),              # one that has no new token
    (28, 4, [61, 30, 1, 17, 33], [61, 100, 1, 400, 33], 128, 700, "head"),  # questions: many row tiles
    (8, 1, [150, 700], [300, 700], 512, 40, "slot"),
    (64, 1, [1, 2, 35], [9, 20, 500], 256, 64, "head"),
    (12, 4, [4, 9], [40, 1000], 16, [1000, 0, 0, 513], "slot"),
    (40, 40, [1] * 3, [40, 50, 600], 16, [i % 7 * 40 for i in range(40)], "head"),
    (7, 1, [90], [1], 8, 300, "head"),                                      # more tokens than slots
    (4, 1, [900, 10], [1000, 10], 64, 5, "head"),                           # an item dealt to many CTAs
]


@pytest.mark.parametrize("dt,flags", [("bf16", 0), ("bf16", SIMT), ("f32", 0)])
@pytest.mark.parametrize("decay", [1.0, 0.75])
@pytest.mark.parametrize("h_q,h_kv,new,lens,page,prefix,order", WEIGH)
def test_weigh(h_q, h_kv, new, lens, page, prefix, order, decay, dt, flags):
    uneven = isinstance(prefix, list)
    b = Batch(sum(lens) + page, h_kv, new, lens, page, dt, order)
    heads, pre = make_prefix(gen(page), prefix if uneven else [prefix] * h_kv, dt, uneven)
    if any(n > x for n, x in zip(new, lens)):
        check_weigh(b, heads, pre, h_q, decay, dt, flags, only_prefix=True)
    else:
        check_weigh(b, heads, pre, h_q, decay, dt, flags)


def check_weigh(b, heads, pre, h_q, decay, dt, flags=0, pad=0, only_prefix=False, lse=None, seed=9):
    T, rows = TYPES[dt], [h[0].shape[0] for h in heads]
    one = all(n == 1 for n in b.new) and not pad
    q = (2 * torch.randn(b.tokens + pad, h_q, D, generator=gen(seed))).to(T)
    if lse is None:  # of an attention over these keys, about
        lse = 3 + math.log(sum(rows) / len(rows) + max(b.lens)) + torch.rand(b.tokens + pad, h_q, generator=gen(3))
        lse[::5, ::3] = -math.inf
    if pad:  # tokens of no sequence
        q[b.tokens:], lse[b.tokens:] = math.nan, math.nan
    pw, w = torch.rand(sum(rows), generator=gen(4)) * 2, torch.rand(b.k.shape[:3], generator=gen(5)) * 2
    dev_pw = pw.cuda() if pre.head_off is not None else pw.view(b.h_kv, -1).cuda()
    # slots that are not in use, and those of the new tokens, hold what there was
    live = torch.zeros(w.shape, dtype=torch.bool)
    old = torch.zeros(w.shape, dtype=torch.bool)
    for s, (n, x) in enumerate(zip(b.new, b.lens)):
        p, r = places(b, s, range(x))
        live[p, :, r] = True
        p, r = places(b, s, range(max(x - n, 0)))
        old[p, :, r] = True
    w[~old] = math.nan
    dev_w = w.cuda()
    ws = E.alloc_weigh_workspace(b.tokens + pad, len(b.new), h_q, b.h_kv, T)
    ws[256:].fill_(255)
    call = lambda x, y: E.weigh(q.cuda(), lse.cuda(), pre, b.cache, x, y, None if one else b.starts.cuda(),  # noqa: E731
                                decay=decay, flags=flags, ws=ws)
    again = dev_pw.clone(), dev_w.clone()
    got = call(dev_pw, dev_w)
    assert got[0] is dev_pw and got[1] is dev_w
    assert E.ecokv_device_status(ws) == (E.ECOKV_OK if not only_prefix else 0)
    new = b.new
    own_k = [k for k, _ in b.own]
    if only_prefix:  # (the definition's masks want slots for all tokens)
        own_k = [torch.zeros(b.h_kv, n, D, dtype=T) for n in new]
    want_p, want_o, size = ref.weigh(q[:b.tokens], lse[:b.tokens], [h[0] for h in heads], own_k, new, 1 / math.sqrt(D))
    rel = (140 * size + 40 + b.tokens * (h_q // b.h_kv) + 10) * U
    x = dev_pw.cpu().view(-1).double()
    want = decay * pw.double() + torch.cat(want_p)
    assert bool(((x - want).abs() <= rel * torch.cat(want_p) + 3 * U * want + 1e-37).all()), \
        float(((x - want).abs() / (rel * torch.cat(want_p) + 3 * U * want + 1e-37)).max())
    y = dev_w.cpu()
    assert torch.equal(y[~live].isnan(), w[~live].isnan())
    if not only_prefix:
        for s, (n, L) in enumerate(zip(new, b.lens)):
            p, r = places(b, s, range(L))
            was = w[p, :, r].double().t()
            was[:, L - n:] = 0.0
            want = decay * was + want_o[s]
            e = (y[p, :, r].double().t() - want).abs()
            assert bool((e <= rel * want_o[s] + 3 * U * want + 1e-37).all()), (s, float(e.max()))
    call(*again)
    assert torch.equal(again[0], dev_pw) and torch.equal(again[1].nan_to_num(9.0), dev_w.nan_to_num(9.0))


@pytest.mark.parametrize("dt,flags", [("bf16", 0), ("bf16", SIMT), ("f32", 0)])
def test_weigh_leaves_out_tokens_of_no_sequence(dt, flags):
    b = Batch(5, 2, [3, 0, 40], [30, 12, 100], 16, dt)
    heads, pre = make_prefix(gen(1), [77, 77], dt, False)
    check_weigh(b, heads, pre, 12, 1.0, dt, flags, pad=9)


@pytest.mark.parametrize("dt,flags", [("bf16", 0), ("bf16", SIMT), ("f32", 0)])
def test_weights_of_an_attention_add_up_to_its_rows(dt, flags):
    """Every row's softmax weights sum to one: what the keys of a head get is its rows."""
    b = Batch(5, 2, [3, 1, 40], [30, 12, 100], 16, dt)
    heads, pre = make_prefix(gen(1), [77, 77], dt, False)
    q = (2 * torch.randn(b.tokens, 12, D, generator=gen(9))).to(TYPES[dt]).cuda()
    lse = torch.empty(b.tokens, 12, device="cuda")
    E.attend(q, pre, b.cache, b.starts.cuda(), lse=lse, flags=flags)
    pw, w = E.weigh(q, lse, pre, b.cache, torch.zeros(2, 77, device="cuda"), torch.zeros(b.k.shape[:3], device="cuda"),
                    b.starts.cuda(), flags=flags)
    total = pw.double().sum(1) + w.double().sum((0, 2))
    # two scores of a weight, of the lse and its own: twice their bound (mag below 60), on 264 rows
    assert bool(((total - 6 * b.tokens).abs() <= 6 * b.tokens * (2 * (140 * 60 + 40) + 1000) * U).all())


@pytest.mark.parametrize("dt,flags", [("bf16", 0), ("bf16", SIMT), ("f32", 0)])
def test_weigh_from_nothing(dt, flags):
    """decay = 0: what the weights were does not count."""
    b = Batch(5, 2, [3, 1, 40], [30, 12, 100], 16, dt)
    heads, pre = make_prefix(gen(1), [300, 300], dt, False)
    q = (2 * torch.randn(b.tokens, 12, D, generator=gen(9))).to(TYPES[dt]).cuda()
    lse = torch.full((b.tokens, 12), 8.0, device="cuda")
    got = [E.weigh(q, lse, pre, b.cache, torch.full((2, 300), x, device="cuda"), torch.full(b.k.shape[:3], x, device="cuda"),
                   b.starts.cuda(), decay=0.0, flags=flags) for x in (0.0, math.nan)]
    assert torch.equal(got[0][0], got[1][0])
    for s, n in enumerate(b.lens):
        p, r = places(b, s, range(n))
        assert torch.equal(got[0][1].cpu()[p, :, r], got[1][1].cpu()[p, :, r])


def test_weigh_without_a_cache_or_a_prefix():
    for dt in ("bf16", "f32"):
        T = TYPES[dt]
        heads, pre = make_prefix(gen(1), [300, 300], dt, False)
        q = (2 * torch.randn(50, 6, D, generator=gen(9))).to(T)
        lse = 9 + torch.rand(50, 6, generator=gen(2))
        pw, none = E.weigh(q.cuda(), lse.cuda(), pre, None, torch.zeros(2, 300, device="cuda"))
        want, _, size = ref.weigh(q, lse, [h[0] for h in heads], [torch.zeros(2, 50, D, dtype=T)], [50], 1 / math.sqrt(D))
        assert none is None
        assert bool(((pw.cpu().double() - torch.stack(want)).abs() <= (140 * size + 250) * U * torch.stack(want) + 1e-37).all())
        # strided weights, another scale
        b = Batch(5, 2, [1] * 3, [30, 12, 100], 16, dt)
        w = torch.zeros(2, 16, b.k.shape[0] + 2, device="cuda").permute(2, 0, 1)[1:-1]
        E.weigh(q[:3].cuda(), lse[:3].cuda(), None, b.cache, None, w, scale=0.05)
        _, want, size = ref.weigh(q[:3], lse[:3], [torch.zeros(0, D)] * 2, [k for k, _ in b.own], b.new, 0.05)
        for s, x in enumerate(want):
            p, r = places(b, s, range(b.lens[s]))
            got = w.cpu()[p, :, r].double().t()
            assert bool(((got - x).abs() <= (140 * size + 100) * U * x + 1e-37).all())
        assert E.weigh(q[:0].cuda(), lse[:0].cuda(), pre, None, pw)[0] is pw


def test_weigh_device_errors():
    """Bad pages, lengths, starts and offsets: a status, and the others' weights as ever."""
    b = Batch(2, 2, [1] * 3, [40, 60, 33], 16, "bf16")
    q = torch.randn(3, 4, D, generator=gen(1)).bfloat16().cuda()
    lse = torch.full((3, 4), 5.0, device="cuda")
    for flags in (0, SIMT):
        good = E.weigh(q, lse, None, b.cache, None, torch.zeros(b.k.shape[:3], device="cuda"), flags=flags)[1]
        for what in ("page", "negative", "length", "starts", "head_off"):
            ws = E.alloc_weigh_workspace(3, 3, 4, 2, torch.bfloat16)
            table, lengths, starts, pre, pw = b.cache.table.clone(), b.cache.lengths.clone(), None, None, None
            if what == "page":
                table[1, 0] = 2 ** 30
            if what == "negative":
                table[1, 1] = -5
            if what == "length":
                lengths[1] = 10 ** 6
                table[1] = table[1, 0]
            if what == "starts":
                starts = ints([0, 1, 0, 3])
            if what == "head_off":
                pre = E.Prefix(*(torch.zeros(10, D, dtype=q.dtype, device="cuda") for _ in range(2)), ints([0, 50, 10]))
                pw = torch.zeros(10, device="cuda")
            w = torch.zeros(b.k.shape[:3], device="cuda")
            E.weigh(q, lse, pre, E.PagedCache(b.dk, b.dv, table, lengths), pw, w, starts, ws=ws, flags=flags)
            assert E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX, what
            if what in ("page", "negative"):
                for s in (0, 2):
                    p, r = places(b, s, range(b.lens[s]))
                    assert torch.equal(w.cpu()[p, :, r], good.cpu()[p, :, r])


def test_weigh_waits_that_run_out():
    """The injected stall: a status, an untouched context, and the next call as ever."""
    b = Batch(2, 2, [1] * 3, [40, 60, 33], 16, "bf16")
    q, lse = torch.randn(3, 4, D, generator=gen(1)).bfloat16().cuda(), torch.full((3, 4), 5.0, device="cuda")
    good = E.weigh(q, lse, None, b.cache, None, torch.zeros(b.k.shape[:3], device="cuda"))[1]
    ws = E.alloc_weigh_workspace(3, 3, 4, 2, torch.bfloat16)
    E.weigh(q, lse, None, b.cache, None, torch.zeros(b.k.shape[:3], device="cuda"), ws=ws, flags=E.ECOKV_FLAG_TEST_STALL,
            timeout_us=2000)
    assert E.ecokv_device_status(ws) == E.ECOKV_ERR_TIMEOUT
    assert torch.equal(E.weigh(q, lse, None, b.cache, None, torch.zeros(b.k.shape[:3], device="cuda"))[1], good)


def test_weigh_refuses_what_does_not_fit():
    b = Batch(1, 2, [1] * 3, [4, 5, 6], 8, "bf16")
    q = torch.zeros(3, 4, D, dtype=torch.bfloat16, device="cuda")
    lse, w = torch.zeros(3, 4, device="cuda"), torch.zeros(b.k.shape[:3], device="cuda")
    for args in ((q.float(), lse, None, b.cache, None, w), (q, lse[:2], None, b.cache, None, w), (q, lse, None, None),
                 (q, lse.double(), None, b.cache, None, w), (q, lse, None, b.cache), (q, lse, None, b.cache, None, w[1:]),
                 (q, lse, None, b.cache, None, w.double()), (q, lse, None, b.cache, None, w.cpu())):
        with pytest.raises((ValueError, TypeError)):
            E.weigh(*args)


# ---------------------------------------------------------------- prune
def run_prune(b, w, budget, limit, first, recent, to_page=0, move="same", alias=True, dt="bf16"):
    """The call and the definition's outcome, compared."""
    T = TYPES[dt]
    B, H = len(b.lens), b.h_kv
    kept = [[None] * H for _ in range(B)]
    for s, n in enumerate(b.lens):
        p, r = places(b, s, range(n))
        for h in range(H):
            kept[s][h] = ref.prune(w[p, h, r], budget, limit, first, recent)
    lens = [len(x[0]) for x in kept]
    if to_page:
        need = [-(-n // to_page) for n in lens]
        perm = torch.randperm(sum(need) + 2, generator=gen(3)).tolist()
        table = torch.full((B, max(need + [1]) + 1), 2 ** 30, dtype=torch.int32)
        for s, n in enumerate(need):
            for c in range(n):
                table[s, c] = perm.pop()
        shape = (sum(need) + 2, H, to_page)
        k, v, ww = torch.full((*shape, D), 5.0, dtype=T), torch.full((*shape, D), 6.0, dtype=T), torch.full(shape, 7.0)
        to = E.PagedCache(k.cuda(), v.cuda(), table.cuda(), torch.zeros(B, dtype=torch.int32, device="cuda"))
    else:
        to_page, table, to = b.page, b.table, None
        k, v, ww = b.k.clone(), b.v.clone(), w.clone()
    for s in range(B):
        for h in range(H):
            at, to_ = places(b, s, kept[s][h]), places(b, s, range(lens[s]), to_page, table)
            for y, z in ((k, b.k), (v, b.v), (ww, w)):
                y[to_[0], h, to_[1]] = z[at[0], h, at[1]]
    dw = w.cuda()
    tw = None if move is None else dw if to is None else torch.full(ww.shape, 7.0, device="cuda")
    idx = torch.full((B, H, limit), 99, dtype=torch.int32, device="cuda")
    out = (b.cache if to is None else to).lengths if alias else None
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    got, ix = E.prune(b.cache, dw, budget, limit, first, recent, to=to, to_weights=tw, lengths_out=out, idx=idx, ws=ws)
    assert ix is idx and E.ecokv_device_status(ws) == 0 and got.tolist() == lens
    want = torch.full((B, H, limit), -1, dtype=torch.int32)
    for s in range(B):
        for h in range(H):
            want[s, h, :lens[s]] = torch.tensor(kept[s][h], dtype=torch.int32)
    assert torch.equal(idx.cpu(), want)
    c = b.cache if to is None else to
    for x, y in ((c.k_pages, k), (c.v_pages, v), (tw, ww)):
        if x is not None:
            assert torch.equal(x.cpu().nan_to_num(123.0), y.nan_to_num(123.0))
    if move is None:
        assert torch.equal(dw.cpu().nan_to_num(9.0), w.nan_to_num(9.0))


PRUNE = [  # h_kv, lengths, page, budget, limit, first, recent
    (2, [9], 8, 8, 8, 1, 2), (4, [100, 3, 0, 64, 65], 16, 20, 64, 4, 8), (3, [300, 299], 32, 1, 1, 0, 0),
    (2, [1000, 4000], 64, 512, 600, 0, 512), (8, [2000] * 5 + [17], 16, 1500, 1999, 4, 32), (1, [40], 4096, 30, 39, 30, 0),
    (4, [500] * 33, 128, 77, 200, 5, 0), (2, [70], 8, 69, 69, 0, 0), (1, [9000], 256, 8000, 8000, 4, 100),
]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("to_page", [0, 8, 64])
@pytest.mark.parametrize("h_kv,lens,page,budget,limit,first,recent", PRUNE)
def test_prune(h_kv, lens, page, budget, limit, first, recent, to_page, dt):
    b = Batch(sum(lens), h_kv, [0] * len(lens), lens, page, dt, "slot" if budget % 2 else "head")
    w = torch.exp(2 * torch.randn(b.k.shape[:3], generator=gen(8)))
    w[w < 0.4] = 0.0  # many equal ones
    run_prune(b, w, budget, limit, first, recent, to_page, move="same" if budget % 3 else None, alias=budget % 4 != 0, dt=dt)


@pytest.mark.parametrize("kind", ["equal", "zeros", "special", "steps", "negative", "tiny"])
def test_prune_of_odd_weights(kind):
    b = Batch(3, 2, [0, 0], [700, 150], 16, "bf16")
    n = b.k.shape[:3]
    w = torch.randn(n, generator=gen(8))
    if kind == "equal":
        w[:] = 3.25
    if kind == "zeros":
        w = torch.where(w > 0, 0.0, -0.0)
    if kind == "special":
        w[w > 1] = math.inf
        w[w < -1] = -math.inf
        w[w.abs() < 0.2] = math.nan
    if kind == "steps":
        w = (w * 2).round()
    if kind == "tiny":
        w = w * 1e-40
    ordered = w.clone()
    if kind == "special":
        # the definition's order: NaN below -inf
        ordered[w == -math.inf] = -3e38
        ordered[w.isnan()] = -math.inf
    kept = [[ref.prune(ordered[places(b, s, range(x))[0], h, places(b, s, range(x))[1]], 100, 120, 3, 5)
             for h in range(2)] for s, x in enumerate(b.lens)]
    _, idx = E.prune(b.cache, w.cuda(), 100, 120, 3, 5)
    for s in range(2):
        for h in range(2):
            assert idx[s, h, :100].tolist() == kept[s][h] and bool((idx[s, h, 100:] == -1).all())


def test_prune_of_a_very_long_sequence():
    """More slots than shared memory keeps keys of; few heads: clusters move the rows."""
    L = 60000
    b = Batch(3, 1, [0], [L], 256, "bf16")
    w = (torch.rand(b.k.shape[:3], generator=gen(8)) * 1000).round()
    run_prune(b, w, 30001, 40000, 4, 1000)


def test_prune_device_errors():
    for what in ("page", "length"):
        b = Batch(3, 2, [0, 0, 0], [50, 60, 30], 16, "bf16")
        w = torch.rand(b.k.shape[:3], generator=gen(8)).cuda()
        good = E.prune(E.PagedCache(b.dk.clone(), b.dv.clone(), b.cache.table, b.cache.lengths), w, 20, 30)[1]
        if what == "page":
            b.cache.table[1, 2] = 2 ** 30
        else:
            b.cache.lengths[1] = 10 ** 7
            b.cache.table[1] = b.cache.table[1, 0]
        ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
        lens, idx = E.prune(b.cache, w, 20, 30, ws=ws)
        assert E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX and lens.tolist() == [20, 20, 30]
        assert torch.equal(idx[0], good[0]) and torch.equal(idx[2], good[2])
        if what == "page":
            assert not bool(((idx[1] >= 32) & (idx[1] < 48)).any())


def test_prune_refuses_what_does_not_fit():
    b = Batch(3, 2, [0, 0], [50, 60], 16, "bf16")
    w = torch.zeros(b.k.shape[:3], device="cuda")
    f = Batch(3, 2, [0, 0], [50, 60], 16, "f32")
    with pytest.raises(TypeError):
        E.prune(b.cache, w, 20, to=f.cache)
    for kw in (dict(weights=w[1:]), dict(weights=w.double()), dict(idx=torch.zeros(2, 2, 20, device="cuda")),
               dict(lengths_out=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(limit=0),
               dict(to=Batch(3, 4, [0, 0], [50, 60], 16, "bf16").cache)):
        with pytest.raises(ValueError):
            E.prune(**dict(dict(cache=b.cache, weights=w, budget=20), **kw))
    for kw in (dict(first=10, recent=11), dict(budget=0, limit=20), dict(limit=10), dict(first=-1)):
        with pytest.raises(E.EcokvError) as e:
            E.prune(**dict(dict(cache=b.cache, weights=w, budget=20), **kw))
        assert e.value.code == E.ECOKV_ERR_INVALID_ARG
