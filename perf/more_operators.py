"""Operators for a cache that shrinks again and for drafted tokens: their cases, plain forms and exact results.

A batch decodes over a shared prefix and paged caches of its own.  Five operators
go with that:

  tree_mask    which drafted tokens each one sees: itself and its ancestors
  attend_tree  attention of every sequence's tree of drafted tokens over the shared
               prefix, its cache and the drafts that the mask lets a token see
  commit       rows of the accepted drafts move to the front, the others' are given up
  weigh        the attention weight that every key of the prefix and the caches gets
               is added to what it has had so far
  prune        eviction from the paged caches by that weight: the heaviest slots, the
               first ones and the last ones stay, in order

Head shapes are those of the repository's workloads (32 x 32, 28/4, 32/8 and the
fp32 8-head layer, d = 128), prefix lengths its budgets and longest prompt, budgets
its own.  Sequence lengths and trees follow from the case alone, so that its work is
known without a seed; values, the order of the pages and the trees whose mask is made
follow from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _cache(name, op, h_q, h_kv, batch, new, kept, page, dtype="bf16", **more):
    """new: the most new tokens (or drafts) of a sequence; kept: the most it has in its cache already."""
    return dict(dict(name=name, op=op, h_q=h_q, h_kv=h_kv, batch=batch, new=new, kept=kept, page=page, dtype=dtype), **more)


def _mask(name, batch, new, words):
    return dict(name=name, op="tree_mask", batch=batch, new=new, words=words)


def _tree(name, h_q, h_kv, batch, new, kept, prefix, page, uneven=False, **more):
    """prefix: rows a head keeps (their mean over the heads where uneven, as under a layer-wide budget)."""
    return _cache(name, "attend_tree", h_q, h_kv, batch, new, kept, page, prefix=prefix, uneven=uneven, **more)


def _commit(name, h_q, h_kv, batch, new, kept, page, weights=False, **more):
    return _cache(name, "commit", h_q, h_kv, batch, new, kept, page, weights=weights, **more)


def _weigh(name, h_q, h_kv, batch, new, kept, prefix, page, uneven=False, decay=1.0, **more):
    return _cache(name, "weigh", h_q, h_kv, batch, new, kept, page, prefix=prefix, uneven=uneven, decay=decay, **more)


def _prune(name, h_q, h_kv, batch, kept, page, budget, limit, first=4, recent=32, to_page=0, **more):
    """to_page: page size of the cache that takes the rows, 0 = the same cache."""
    return _cache(name, "prune", h_q, h_kv, batch, 1, kept, page, budget=budget, limit=limit, first=first, recent=recent,
                  to_page=to_page, **more)


def listed():
    return [
        # the drafts of one sequence
        _mask("mask_1", 1, 25, 1),
        # a large batch with wide trees
        _mask("mask_64", 64, 256, 4),
        # one user's answer about an image, a small tree of drafts
        _tree("tree_image_1", 32, 8, 1, 25, 40, 205, 16),
        # answers about one video verified together
        _tree("tree_video_16", 28, 4, 16, 61, 500, 3277, 16),
        # the fp32 layer
        _tree("tree_f32", 8, 8, 8, 13, 200, 128, 16, dtype="f32"),
        # the accepted drafts of that video batch
        _commit("commit_video_16", 28, 4, 16, 61, 500, 16),
        # wide trees, long caches with weights of their own, the fp32 layer
        _commit("commit_f32_64", 8, 8, 64, 256, 2000, 64, weights=True, dtype="f32"),
        # one decode step of the fp32 layer, older weights fading
        _weigh("weigh_f32", 8, 8, 8, 3, 200, 128, 16, decay=0.9, dtype="f32"),
        # one decode step of many long answers: the pages dominate
        _weigh("weigh_pages_64", 28, 4, 64, 1, 4096, 1024, 64, uneven=True),
        # the batch's questions at once over the video at the larger budget
        _weigh("weigh_questions", 28, 4, 16, 61, 100, 6554, 32),
        # the fp32 layer's sequences past 300 slots go to 205 in a smaller pool
        _prune("prune_f32_pool", 8, 8, 5, 1500, 16, 205, 300, to_page=32, dtype="f32"),
        # many long answers back to 1024 slots where they are
        _prune("prune_pages_64", 28, 4, 64, 4096, 64, 1024, 1024),
    ]


def _logu(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / (5 if c.get("dtype") == "f32" else 50))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        del c["name"]
        if _cost(c) <= most:
            return c


def _draw(rng):
    op = rng.choice(["tree_mask", "attend_tree", "attend_tree", "commit", "weigh", "weigh", "prune", "prune"])
    if op == "tree_mask":
        new = _logu(rng, 8, 512)  # (a tree of one token has one mask)
        return _mask("", _logu(rng, 1, 64), new, -(-new // 64) + rng.randint(0, 1))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    h_q, h_kv = rng.choice([(32, 32), (28, 4), (32, 8), (8, 8), (28, 4)])
    page = rng.choice([8, 16, 16, 32, 64, 128, 256])
    batch = _logu(rng, 1, 64)
    kept = _logu(rng, 1, 4096)
    prefix = 0 if rng.random() < 0.1 else _logu(rng, 1, 16384 if dtype == "f32" else 131072)
    uneven = rng.random() < 0.3
    if op == "attend_tree":
        return _tree("", h_q, h_kv, batch, _logu(rng, 1, 256), kept, prefix, page, uneven, dtype=dtype)
    if op == "commit":
        return _commit("", h_q, h_kv, batch, _logu(rng, 1, 256), kept, page, rng.random() < 0.5, dtype=dtype)
    if op == "weigh":
        new = 1 if rng.random() < 0.6 else _logu(rng, 2, 64)
        return _weigh("", h_q, h_kv, batch, new, kept, prefix, page, uneven, rng.choice([1.0, 1.0, 0.9]), dtype=dtype)
    kept = _logu(rng, 64, 16384)
    budget = _logu(rng, 16, max(16, kept // 2))
    first, recent = rng.choice([0, 1, 4]), rng.randint(0, budget // 4)
    return _prune("", h_q, h_kv, batch, kept, page, budget, budget + rng.choice([0, 0, 16, budget // 2]), first, recent,
                  rng.choice([0, 0, 16, 32, 128]), dtype=dtype)


def _ragged(c):
    """(new tokens, slots in use with them) of every sequence: from the case alone."""
    rng = random.Random("%d %d %d" % (c["batch"], c["new"], c.get("kept", 0)))
    new = [rng.randint((c["new"] + 1) // 2, c["new"]) for _ in range(c["batch"])]
    kept = [rng.randint(0, c.get("kept", 0)) for _ in range(c["batch"])]
    new[0], kept[0] = c["new"], c.get("kept", 0)
    return new, [n + k for n, k in zip(new, kept)]


def _trees(c, seed=0):
    """Every sequence's drafts: the parent of each, -1 where it follows the last token of the cache."""
    rng = random.Random("trees %d %d %d" % (c["batch"], c["new"], seed))
    out = []
    for n in _ragged(c)[0]:
        # half of the drafts go on from one of the last few, the others from any: chains with branches
        out.append([-1 if i == 0 or rng.random() < 0.05 else rng.randint(max(0, i - 4), i - 1) if rng.random() < 0.5
                    else rng.randint(0, i - 1) for i in range(n)])
    return out


def _paths(c):
    """The drafts that are accepted: a path from a root, its length up to the leaf."""
    rng = random.Random("paths %d %d" % (c["batch"], c["new"]))
    out = []
    for parents in _trees(c):
        at, path = rng.randrange(len(parents)), []
        while at >= 0:
            path.append(at)
            at = parents[at]
        path.reverse()
        out.append(path[:rng.randint(0, len(path))] if rng.random() < 0.5 else path)
    return out


def _prefix_rows(c):
    """Prefix rows of every KV head: the layer-wide budget gives some heads 1.6 times the mean and others 0.4."""
    P, H = c["prefix"], c["h_kv"]
    rows = [P] * H
    if c["uneven"]:
        for h in range(0, H - 1, 2):
            s = (3 + h % 4) * P // 10
            rows[h], rows[h + 1] = P + s, P - s
    return rows


def work(c):
    new, lens = _ragged(c)
    tokens = sum(new)
    if c["op"] == "tree_mask":
        return {"bytes": tokens * (4 + 8 * c["words"]) + 4 * (c["batch"] + 1), "flops": 0}
    e = 4 if c["dtype"] == "f32" else 2
    h_q, h_kv = c["h_q"], c["h_kv"]
    pages = sum(-(-x // c["page"]) for x in lens)
    if c["op"] == "attend_tree":
        rows = sum(_prefix_rows(c))
        drafts = sum(_seen(parents) for parents in _trees(c))
        pairs = tokens * (h_q // h_kv) * rows + h_q * (sum(n * (x - n) for n, x in zip(new, lens)) + drafts)
        return {"bytes": 2 * (rows + h_kv * sum(lens)) * D * e + 2 * tokens * h_q * D * e + 8 * tokens * -(-c["new"] // 64)
                + 4 * pages + 8 * c["batch"], "flops": 4 * D * pairs}
    if c["op"] == "commit":
        paths = _paths(c)
        moved = sum(i != s for p in paths for i, s in enumerate(p)) * h_kv
        return {"bytes": moved * (4 * D * e + (8 if c["weights"] else 0)) + 4 * sum(len(p) for p in paths) + 16 * c["batch"],
                "flops": 0}
    if c["op"] == "weigh":
        rows = sum(_prefix_rows(c))
        pairs = tokens * (h_q // h_kv) * rows + h_q * sum(n * x - n * (n - 1) // 2 for n, x in zip(new, lens))
        return {"bytes": (rows + h_kv * sum(lens)) * (D * e + 8) - 4 * h_kv * tokens + tokens * h_q * (D * e + 4) + 4 * pages
                + 8 * c["batch"], "flops": 2 * D * pairs}
    # rows that stay where they are in the same cache are not moved
    cut = [x for x in lens if x > c["limit"]]
    if c["to_page"]:
        rows = sum(c["budget"] if x > c["limit"] else x for x in lens)
    else:
        rows = len(cut) * (c["budget"] - min(c["first"], c["budget"]))
    return {"bytes": h_kv * (4 * sum(cut) + rows * (4 * D * e + (8 if c["to_page"] else 0)) + 4 * c["batch"] * c["limit"])
            + 4 * pages + 8 * c["batch"], "flops": 0}


def _seen(parents):
    """Drafts that a tree's tokens see, themselves among them."""
    depth = []
    for p in parents:
        depth.append(1 if p < 0 else depth[p] + 1)
    return sum(depth)


# ---------------------------------------------------------------- inputs
def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _table(lens, page, order):
    """[batch][pages a sequence, one spare] of the pool's pages in the given order."""
    need = torch.tensor([-(-x // page) for x in lens])
    cols = int(need.max()) + 1
    used = torch.cat([torch.zeros(1, dtype=torch.int64), need.cumsum(0)])
    inside = torch.arange(cols) < need[:, None]
    at = torch.where(inside, used[:-1, None] + torch.arange(cols), 0)
    return torch.where(inside.to(DEV), order[at.to(DEV)], torch.zeros((), dtype=torch.int32, device=DEV)).contiguous()


def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rnd = lambda *n: torch.randn(*n, generator=g, device=DEV)  # noqa: E731
    s = {"case": c}
    new, lens = _ragged(c)
    tokens = sum(new)
    s["starts"] = _ints([0] + new).cumsum(0).int()
    s["batch_max"] = max(new)
    if c["op"] in ("tree_mask", "attend_tree"):
        trees = _trees(c, int(seed) if c["op"] == "tree_mask" else 0)
        s["parents"] = _ints([p for t in trees for p in t])
    if c["op"] == "tree_mask":
        s["mask"] = torch.zeros(tokens, c["words"], dtype=torch.int64, device=DEV)
        return s
    dt, h_q, h_kv, page = TYPES[c["dtype"]], c["h_q"], c["h_kv"], c["page"]
    # a pool of pages that the sequences hold in any order, some of it free
    n_pages = sum(-(-x // page) for x in lens) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).int()
    s["table"], s["lengths"] = _table(lens, page, order), _ints(lens)
    s["len_max"], s["step"] = max(lens), c["new"] == 1
    # keys in a narrow cone; [page][head][slot][d], slots that no sequence has reached hold what was there before
    u = rnd(h_kv, D)
    u = u / torch.linalg.vector_norm(u, dim=1, keepdim=True)
    s["k_pages"] = (4.0 * u[:, None] + rnd(n_pages, h_kv, page, D)).to(dt)
    if c["op"] != "weigh":
        s["v_pages"] = rnd(n_pages, h_kv, page, D).to(dt)
    else:  # (values play no part)
        s["v_pages"] = s["k_pages"]
    if c["op"] == "commit":
        paths = _paths(c)
        most = max(len(p) for p in paths) + 1
        s["accepted"] = _ints([p + [0] * (most - len(p)) for p in paths])
        s["counts"] = _ints([len(p) for p in paths])
        s["weights"] = rnd(n_pages, h_kv, page).abs() if c["weights"] else None
        s["lengths_out"] = torch.zeros_like(s["lengths"])
    elif c["op"] == "prune":
        # weights as they are after a while: a few heavy slots, many light ones, some that nothing has looked at
        s["weights"] = torch.exp(2.0 * rnd(n_pages, h_kv, page) - 4.0) * (rnd(n_pages, h_kv, page) > -1.0)
        s["lengths_out"] = torch.zeros_like(s["lengths"])
        s["idx"] = torch.zeros(c["batch"], h_kv, c["limit"], dtype=torch.int32, device=DEV)
        if c["to_page"]:
            kept = [c["budget"] if x > c["limit"] else x for x in lens]
            n_to = sum(-(-x // c["to_page"]) for x in kept) + 1
            s["to_table"] = _table(kept, c["to_page"], torch.randperm(n_to, generator=g, device=DEV).int())
            s["to_k"], s["to_v"] = (torch.zeros(n_to, h_kv, c["to_page"], D, dtype=dt, device=DEV) for _ in range(2))
            s["to_weights"] = torch.zeros(n_to, h_kv, c["to_page"], device=DEV)
    else:
        s["q"] = (4.0 * u.repeat_interleave(h_q // h_kv, 0) + rnd(tokens, h_q, D)).to(dt)
        rows = _prefix_rows(c)
        s["prefix_off"], s["row_max"] = _ints([0] + rows).cumsum(0).int(), max(rows)
        if c["uneven"]:
            head = torch.repeat_interleave(torch.arange(h_kv), torch.tensor(rows)).to(DEV)
            s["prefix_k"] = (4.0 * u[head] + rnd(sum(rows), D)).to(dt)
        else:
            s["prefix_k"] = (4.0 * u[:, None] + rnd(h_kv, rows[0], D)).to(dt)
        if c["op"] == "attend_tree":
            s["prefix_v"] = rnd(*s["prefix_k"].shape).to(dt)
            words = -(-c["new"] // 64)
            s["mask"] = _pack(_reach(s), s, words)
            s["out"] = torch.empty(tokens, h_q, D, dtype=dt, device=DEV)
            s["lse"] = torch.empty(tokens, h_q, device=DEV)
        else:
            s["prefix_v"] = s["prefix_k"]
            s["lse"] = torch.empty(tokens, h_q, device=DEV)
            _step_lse(s)
            s["weights"] = rnd(n_pages, h_kv, page).abs()
            s["prefix_weights"] = rnd(*s["prefix_k"].shape[:-1]).abs()
    if own:  # the handles and the workspace that a program keeps for a model and its cache
        from paper_2609_06663_gb300 import ecokv as E
        s["cache"] = E.PagedCache(s["k_pages"], s["v_pages"], s["table"], s["lengths"])
        if c["op"] in ("attend_tree", "weigh"):
            s["prefix"] = E.Prefix(s["prefix_k"], s["prefix_v"], s["prefix_off"] if c["uneven"] else None)
            alloc = E.alloc_attend_workspace if c["op"] == "attend_tree" else E.alloc_weigh_workspace
            s["ws"] = alloc(tokens, c["batch"], h_q, h_kv, dt)
        if c.get("to_page"):
            s["to"] = E.PagedCache(s["to_k"], s["to_v"], s["to_table"], s["lengths_out"])
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    return (_run_own if own else _run_plain)[s["case"]["op"]](s)


def _own_mask(s):
    from paper_2609_06663_gb300 import ecokv as E
    return E.tree_mask(s["parents"], s["starts"], mask=s["mask"])


def _own_tree(s):
    from paper_2609_06663_gb300 import ecokv as E
    out = E.attend_tree(s["q"], s["prefix"], s["cache"], s["mask"], s["starts"], out=s["out"], lse=s["lse"], ws=s["ws"])
    return out, s["lse"]


def _own_commit(s):
    from paper_2609_06663_gb300 import ecokv as E
    n = E.commit(s["cache"], s["accepted"], s["counts"], s["starts"], weights=s["weights"], lengths_out=s["lengths_out"])
    return (n, s["k_pages"], s["v_pages"]) + (() if s["weights"] is None else (s["weights"],))


def _own_weigh(s):
    from paper_2609_06663_gb300 import ecokv as E
    E.weigh(s["q"], s["lse"], s["prefix"], s["cache"], s["prefix_weights"], s["weights"],
            starts=None if s["step"] else s["starts"], decay=s["case"]["decay"], ws=s["ws"])
    return s["prefix_weights"], s["weights"]


def _own_prune(s):
    from paper_2609_06663_gb300 import ecokv as E
    c, to = s["case"], s.get("to")
    n, idx = E.prune(s["cache"], s["weights"], c["budget"], c["limit"], c["first"], c["recent"], to=to,
                     to_weights=s.get("to_weights"), lengths_out=s["lengths_out"], idx=s["idx"])
    return (n, idx, s["k_pages"], s["v_pages"]) if to is None else (n, idx, s["to_k"], s["to_v"], s["to_weights"])


def _places(s):
    """(sequence, number within it) of every new token."""
    starts = s["starts"].long()
    t = torch.arange(int(s["parents"].shape[0] if "parents" in s else s["q"].shape[0]), device=DEV)
    b = torch.searchsorted(starts, t, right=True) - 1
    return b, t - starts[b]


def _reach(s):
    """[batch, T, T]: draft j is draft i or one of its ancestors."""
    b, i = _places(s)
    B, T = s["starts"].shape[0] - 1, s["batch_max"]
    up = torch.zeros(B, T, T, device=DEV)
    has = (s["parents"] >= 0).float()
    up[b, i, s["parents"].long().clamp(min=0)] = has
    up = up + torch.eye(T, device=DEV)
    for _ in range(max(1, (T - 1).bit_length())):  # twice as far each time
        up = ((up @ up) > 0).float()
    return up > 0


def _pack(reach, s, words):
    b, i = _places(s)
    seen = torch.zeros(b.shape[0], 64 * words, dtype=torch.int64, device=DEV)
    seen[:, :reach.shape[2]] = reach[b, i].long()
    return (seen.view(-1, words, 64) << torch.arange(64, device=DEV)).sum(-1)  # (distinct powers of two: no carries)


def _plain_mask(s):
    s["mask"].copy_(_pack(_reach(s), s, s["case"]["words"]))
    return s["mask"]


def _batch_keys(s, x):
    """The caches' rows as rectangles [B, h_kv, L, D] in 32 bits."""
    c, L = s["case"], s["len_max"]
    cols = -(-L // c["page"])
    x = x[s["table"][:, :cols].long()].transpose(1, 2).reshape(c["batch"], c["h_kv"], cols * c["page"], D)[:, :, :L].float()
    live = torch.arange(L, device=DEV) < s["lengths"][:, None]
    return torch.where(live[:, None, :, None], x, torch.zeros((), device=DEV))


def _batch_rows(s):
    """The new tokens' queries as rectangles [B, h_kv, T, g, D] in 32 bits, scaled."""
    c = s["case"]
    b, i = _places(s)
    q = torch.zeros(c["batch"], s["batch_max"], c["h_q"], D, device=DEV)
    q[b, i] = s["q"].float() / math.sqrt(D)
    return q.view(c["batch"], s["batch_max"], c["h_kv"], -1, D).transpose(1, 2)


def _own_seen(s):
    """[B, T, L]: what a new token sees of its sequence's slots."""
    slot = torch.arange(s["len_max"], device=DEV)
    base = s["lengths"] - (s["starts"][1:] - s["starts"][:-1])
    if "mask" not in s:
        return slot <= (base[:, None] + torch.arange(s["batch_max"], device=DEV))[..., None]
    b, i = _places(s)
    draft = slot - base[:, None]  # [B, L]
    words = s["mask"].shape[1]
    at = draft.clamp(0, 64 * words - 1)[b]  # [tokens, L]
    bit = (s["mask"].gather(1, at // 64) >> (at % 64)) & 1
    seen = torch.zeros(s["case"]["batch"], s["batch_max"], s["len_max"], dtype=torch.bool, device=DEV)
    seen[b, i] = (draft[b] < 0) | ((bit == 1) & (slot < s["lengths"][b][:, None]))
    return seen


def _prefix_heads(s):
    """Every head's (first row, rows): known to the host, as the call's sizes are."""
    at, out = 0, []
    for n in _prefix_rows(s["case"]):
        out.append((at, n))
        at += n
    return out


def _scores(s):
    """([h_kv] scores [tokens * g, rows] of the prefix, scores [B, h_kv, T, g, L] of the caches, -inf where unseen)."""
    c = s["case"]
    g, tokens = c["h_q"] // c["h_kv"], s["q"].shape[0]
    qh = (s["q"].float() / math.sqrt(D)).view(tokens, c["h_kv"], g, D).transpose(0, 1).reshape(c["h_kv"], tokens * g, D)
    k = s["prefix_k"].reshape(-1, D)
    sp = [qh[h] @ k[r:r + n].float().t() for h, (r, n) in enumerate(_prefix_heads(s))]
    qb, kb = _batch_rows(s), _batch_keys(s, s["k_pages"])
    B, H, T = qb.shape[:3]
    so = (qb.reshape(B, H, T * g, D) @ kb.transpose(2, 3)).view(B, H, T, g, -1)
    return sp, torch.where(_own_seen(s)[:, None, :, None], so, torch.full((), float("-inf"), device=DEV))


def _tops(s, sp, so):
    """Largest score of every row [tokens, h_kv, g], and the caches' scores by token [tokens, h_kv, g, L]."""
    c = s["case"]
    b, i = _places(s)
    so = so.transpose(1, 2)[b, i]  # [tokens, h_kv, g, L]
    top = so.amax(-1)
    if c["prefix"]:
        top = torch.maximum(top, torch.stack([x.amax(-1).view(-1, so.shape[2]) if x.shape[1] else
                                              torch.full((so.shape[0], so.shape[2]), float("-inf"), device=DEV)
                                              for x in sp], 1))
    return top, so


def _plain_tree(s):
    c = s["case"]
    g, tokens = c["h_q"] // c["h_kv"], s["q"].shape[0]
    b, i = _places(s)
    sp, so = _scores(s)
    top, so = _tops(s, sp, so)
    eo = torch.exp(so - top[..., None])
    total, out = eo.sum(-1), torch.zeros(tokens, c["h_kv"], g, D, device=DEV)
    v = s["prefix_v"].reshape(-1, D)
    for h, (r, n) in enumerate(_prefix_heads(s)):
        e = torch.exp(sp[h] - top[:, h].reshape(-1, 1))
        total[:, h] += e.sum(-1).view(tokens, g)
        out[:, h] = (e @ v[r:r + n].float()).view(tokens, g, D)
    eb = torch.zeros(c["batch"], s["batch_max"], c["h_kv"], g, s["len_max"], device=DEV)
    eb[b, i] = eo
    eb = eb.transpose(1, 2).reshape(c["batch"], c["h_kv"], -1, s["len_max"])
    ob = (eb @ _batch_keys(s, s["v_pages"])).view(c["batch"], c["h_kv"], s["batch_max"], g, D)
    out = out + ob.transpose(1, 2)[b, i]
    lse = (top + torch.log(total)).reshape(tokens, c["h_q"])
    return (out / total[..., None]).reshape(tokens, c["h_q"], D).to(s["q"].dtype), lse


def _step_lse(s):
    """The rows' logarithms of sums of exponentials, as the attention before has left them."""
    c = s["case"]
    sp, so = _scores(s)
    top, so = _tops(s, sp, so)
    total = torch.exp(so - top[..., None]).sum(-1)
    for h in range(c["h_kv"]):
        total[:, h] += torch.exp(sp[h] - top[:, h].reshape(-1, 1)).sum(-1).view(-1, total.shape[2])
    s["lse"].copy_((top + torch.log(total)).reshape(s["lse"].shape))


def _live(s):
    """(sequence, slot, page, row) of every slot in use."""
    page = s["case"]["page"]
    b, slot = torch.nonzero(torch.arange(s["len_max"], device=DEV) < s["lengths"][:, None], as_tuple=True)
    return b, slot, s["table"].long()[b, slot // page], slot % page


def _plain_weigh(s):
    c = s["case"]
    g, tokens = c["h_q"] // c["h_kv"], s["q"].shape[0]
    b, i = _places(s)
    sp, so = _scores(s)
    lse = s["lse"].view(tokens, c["h_kv"], g)
    pw = s["prefix_weights"].view(-1)
    for h, (r, n) in enumerate(_prefix_heads(s)):
        pw[r:r + n] = c["decay"] * pw[r:r + n] + torch.exp(sp[h] - lse[:, h].reshape(-1, 1)).sum(0)
    lb = torch.zeros(c["batch"], s["batch_max"], c["h_kv"], g, device=DEV)
    lb[b, i] = lse
    w = torch.exp(so - lb.transpose(1, 2)[..., None])
    there = torch.arange(s["batch_max"], device=DEV) < (s["starts"][1:] - s["starts"][:-1])[:, None]
    w = torch.where(there[:, None, :, None, None], w, torch.zeros((), device=DEV)).sum((2, 3))  # [B, h_kv, L]
    b, slot, page, row = _live(s)
    base = (s["lengths"] - (s["starts"][1:] - s["starts"][:-1]))[b]
    was = torch.where((slot < base)[:, None], s["weights"][page, :, row], torch.zeros((), device=DEV))
    s["weights"][page, :, row] = c["decay"] * was + w.transpose(1, 2)[b, slot]
    return s["prefix_weights"], s["weights"]


def _plain_commit(s):
    page, table = s["case"]["page"], s["table"].long()
    base = s["lengths"] - (s["starts"][1:] - s["starts"][:-1])
    b, i = torch.nonzero(torch.arange(s["accepted"].shape[1], device=DEV) < s["counts"][:, None], as_tuple=True)
    src, dst = base[b] + s["accepted"][b, i], base[b] + i
    at, to = table[b, src // page], table[b, dst // page]
    out = [s["k_pages"], s["v_pages"]] + ([] if s["weights"] is None else [s["weights"]])
    for x in out:
        x[to, :, dst % page] = x[at, :, src % page]
    s["lengths_out"].copy_(base + s["counts"])
    return (s["lengths_out"], *out)


def _plain_prune(s):
    c = s["case"]
    page, H, L, lens = c["page"], c["h_kv"], s["len_max"], s["lengths"].long()
    keep = torch.where(lens > c["limit"], torch.full((), c["budget"], device=DEV), lens)
    cols = -(-L // page)
    w = s["weights"][s["table"][:, :cols].long()].transpose(1, 2).reshape(c["batch"], H, cols * page)[..., :L]
    slot = torch.arange(L, device=DEV)
    # the first and the last ones before all others, slots past the length behind them; equal ones in their order
    fixed = (slot < c["first"]) | (slot >= lens[:, None] - c["recent"])
    w = torch.where(fixed[:, None], torch.full((), float("inf"), device=DEV), w)
    w = torch.where((slot < lens[:, None])[:, None], w, torch.full((), float("-inf"), device=DEV))
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    place = torch.empty_like(order)
    place.scatter_(-1, order, slot.expand_as(order).contiguous())
    b, h, at = torch.nonzero(place < keep[:, None, None], as_tuple=True)  # slots that stay, in order
    i = (place < keep[:, None, None]).cumsum(-1)[b, h, at] - 1
    s["idx"].fill_(-1)
    s["idx"][b, h, i] = at.int()
    table, to_page, to_table = s["table"].long(), page, s["table"].long()
    names = [("k_pages", "k_pages"), ("v_pages", "v_pages")]
    if c["to_page"]:
        to_page, to_table = c["to_page"], s["to_table"].long()
        names = [("k_pages", "to_k"), ("v_pages", "to_v"), ("weights", "to_weights")]
    for x, y in names:
        s[y][to_table[b, i // to_page], h, i % to_page] = s[x][table[b, at // page], h, at % page]
    s["lengths_out"].copy_(keep)
    return (s["lengths_out"], s["idx"], *(s[y] for _, y in names))


_run_own = {"tree_mask": _own_mask, "attend_tree": _own_tree, "commit": _own_commit, "weigh": _own_weigh,
            "prune": _own_prune}
_run_plain = {"tree_mask": _plain_mask, "attend_tree": _plain_tree, "commit": _plain_commit, "weigh": _plain_weigh,
              "prune": _plain_prune}


# ---------------------------------------------------------------- from the definitions, in 64 bits
def exact(c, seed):
    s = prepare(c, seed)
    return {"tree_mask": _exact_mask, "attend_tree": _exact_rows, "weigh": _exact_rows, "commit": _exact_commit,
            "prune": _exact_prune}[c["op"]](c, s)


def _exact_mask(c, s):
    parents, starts, out = s["parents"].tolist(), s["starts"].tolist(), []
    for t0, t1 in zip(starts, starts[1:]):
        for i in range(t1 - t0):
            bits, at = 0, i
            while at >= 0:
                bits |= 1 << at
                at = parents[t0 + at]
            words = [(bits >> (64 * w)) & (2 ** 64 - 1) for w in range(c["words"])]
            out.append([x - 2 ** 64 if x >= 2 ** 63 else x for x in words])
    return torch.tensor(out, dtype=torch.int64, device=DEV)


def _rows_of(s, x, b, n):
    """Slots 0 .. n - 1 of sequence b: (page, row) and the rows [n, h_kv, ...] of x."""
    slot = torch.arange(n, device=DEV)
    page, row = s["table"][b, slot // s["case"]["page"]].long(), slot % s["case"]["page"]
    return page, row, x[page, :, row]


def _exact_rows(c, s):
    """Attention and the weights of its keys, sequence by sequence and head by head."""
    if work(c)["flops"] > 3e12:
        return None
    tree = c["op"] == "attend_tree"
    new, lens = _ragged(c)
    g, H = c["h_q"] // c["h_kv"], c["h_kv"]
    off = [0]
    for n in _prefix_rows(c):
        off.append(off[-1] + n)
    pk, pv = s["prefix_k"].reshape(-1, D), s["prefix_v"].reshape(-1, D)
    tokens = sum(new)
    out, lse = torch.zeros(tokens, c["h_q"], D, dtype=torch.float64, device=DEV), s["lse"].double().clone()
    if not tree:
        prefix_weights, weights = s["prefix_weights"].double().view(-1) * c["decay"], s["weights"].double()
    trees = _trees(c) if tree else None
    t = 0
    for b, (n, x) in enumerate(zip(new, lens)):
        seen = torch.ones(n, x, dtype=torch.bool)
        if tree:
            seen[:, x - n:] = False
            for i in range(n):
                at = i
                while at >= 0:
                    seen[i, x - n + at] = True
                    at = trees[b][at]
        else:
            seen[:, x - n:] = torch.tril(torch.ones(n, n, dtype=torch.bool))
        seen = seen.to(DEV)
        page, row, k = _rows_of(s, s["k_pages"], b, x)
        v = _rows_of(s, s["v_pages"], b, x)[2]
        for h in range(H):
            q = s["q"][t:t + n, h * g:(h + 1) * g].double()
            sp = torch.einsum("ngd,kd->ngk", q, pk[off[h]:off[h + 1]].double()) * D ** -0.5
            so = torch.einsum("ngd,kd->ngk", q, k[:, h].double()) * D ** -0.5
            so = so.masked_fill(~seen[:, None], float("-inf"))
            if tree:
                score = torch.cat([sp, so], -1)
                lse[t:t + n, h * g:(h + 1) * g] = torch.logsumexp(score, -1)
                p = torch.softmax(score, -1)
                both = torch.cat([pv[off[h]:off[h + 1]], v[:, h]]).double()
                out[t:t + n, h * g:(h + 1) * g] = torch.einsum("ngk,kd->ngd", p, both)
            else:
                at = lse[t:t + n, h * g:(h + 1) * g, None]
                prefix_weights[off[h]:off[h + 1]] += torch.exp(sp - at).sum((0, 1))
                was = weights[page, h, row] * c["decay"]
                was[x - n:] = 0.0
                weights[page, h, row] = was + torch.exp(so - at).sum((0, 1))
        t += n
    return (out, lse) if tree else (prefix_weights.view(s["prefix_weights"].shape), weights)


def _exact_commit(c, s):
    new, lens = _ragged(c)
    paths = _paths(c)
    out = [s["k_pages"].double(), s["v_pages"].double()] + ([] if s["weights"] is None else [s["weights"].double()])
    for b, (n, x, path) in enumerate(zip(new, lens, paths)):
        page, row, _ = _rows_of(s, s["k_pages"], b, x)
        for i, p in enumerate(path):  # (a path ascends: no row is written before it is read)
            for y in out:
                y[page[x - n + i], :, row[x - n + i]] = y[page[x - n + p], :, row[x - n + p]].clone()
    return (_ints([x - n + len(p) for n, x, p in zip(new, lens, paths)]), *out)


def _exact_prune(c, s):
    lens = _ragged(c)[1]
    idx = torch.full((c["batch"], c["h_kv"], c["limit"]), -1, dtype=torch.int32)
    keep = [c["budget"] if x > c["limit"] else x for x in lens]
    if c["to_page"]:
        names = [("k_pages", "to_k"), ("v_pages", "to_v"), ("weights", "to_weights")]
    else:
        names = [("k_pages", "k_pages"), ("v_pages", "v_pages")]
    out = [s[y].double() for _, y in names]
    for b, (x, n) in enumerate(zip(lens, keep)):
        page, row, w = _rows_of(s, s["weights"], b, x)
        w = w.t().double().cpu().numpy()
        i = torch.arange(n, device=DEV)
        to_page = c["to_page"] or c["page"]
        to = (s["to_table"] if c["to_page"] else s["table"])[b, i // to_page].long()
        for h in range(c["h_kv"]):
            stay = list(range(x))
            if x > c["limit"]:
                lo, hi = c["first"], x - c["recent"]
                best = lo + np.argsort(-w[h, lo:hi], kind="stable")[:n - lo - (x - hi)]
                stay = list(range(lo)) + sorted(best.tolist()) + list(range(hi, x))
            idx[b, h, :n] = torch.tensor(stay, dtype=torch.int32)
            at = torch.tensor(stay, dtype=torch.int64, device=DEV)
            for y, (src, _) in zip(out, names):
                y[to, h, i % to_page] = s[src][page[at], h, row[at]].double()
    return (_ints(keep), idx.to(DEV), *out)
