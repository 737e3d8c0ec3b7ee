"""The operators of a decode step over an evicted cache: their cases, plain forms and exact results.

After the eviction pass a prompt's keys and values are a compact prefix
[h_kv][kept][d]; a batch of sequences that share it (several questions about the
same video) then grows caches of its own, in pages.  Three operators do that:

  rotate   norm of each query and key head (optional) and rotary positions
  append   the same on the way of new keys and values into the paged cache
  attend   attention of the batch over the shared prefix and its own pages

Head shapes are those of the repository's workloads (32 x 32, 28/4, 32/8 and the
fp32 8-head layer, d = 128), prefix lengths its budgets (205, 1024, 3277, 6554,
13107) and longest prompt (131072).  Sequence lengths are ragged and follow from
the case alone, so that its work is known without a seed; values and the order
of the pages follow from the seed.
"""
import math
import random

import torch

own = False

D = 128
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rot(name, h_q, h_kv, tokens, dtype="bf16", layout="half", rot=128, axes=1, norm=False, base=1e6, scaling="none",
         factor=1.0, first=0, **more):
    c = dict(name=name, op="rotate", h_q=h_q, h_kv=h_kv, tokens=tokens, dtype=dtype, layout=layout, rot=rot, axes=axes,
             norm=norm, base=base, scaling=scaling, factor=factor, first=first)
    return dict(c, **more)


def _append(name, h_q, h_kv, batch, new, kept, page, **more):
    """new: the most new tokens of a sequence; kept: the most it has in its cache already."""
    c = _rot(name, h_q, h_kv, 0, **more)
    del c["tokens"]
    return dict(c, op="append", batch=batch, new=new, kept=kept, page=page)


def _attend(name, h_q, h_kv, batch, new, kept, prefix, page, dtype="bf16", uneven=False):
    """prefix: rows a head keeps (their mean over the heads where uneven, as under a layer-wide budget)."""
    return dict(name=name, op="attend", h_q=h_q, h_kv=h_kv, batch=batch, new=new, kept=kept, prefix=prefix, page=page,
                dtype=dtype, uneven=uneven)


def listed():
    return [
        # one decoded token of one sequence: norms and rotation of a single row per head
        _rot("rotate_token_norm", 32, 8, 1, layout="interleaved", rot=64, norm=True, base=1e4, first=4099),
        # a video prompt's queries and keys with time, height and width positions
        _rot("rotate_prompt_32k", 28, 4, 32768, axes=3),
        # the fp32 layer past the length its frequencies were made for, part of the head rotated
        _rot("rotate_f32_yarn", 8, 8, 5003, dtype="f32", rot=96, norm=True, base=1e4, scaling="yarn", factor=8.0,
             first=60000),
        # one decode step of a small batch
        _append("append_step", 28, 4, 16, 1, 300, 16, axes=3, first=32768),
        # the questions themselves enter the cache, of odd lengths
        _append("append_questions", 32, 8, 48, 301, 77, 64, norm=True, first=8192),
        # the first decoded tokens after an image prompt (205 rows a head kept)
        _attend("attend_image_4", 32, 32, 4, 1, 40, 205, 16),
        # a batch of answers about one video, ragged caches of their own
        _attend("attend_video_16", 28, 4, 16, 1, 500, 3277, 16),
        # the batch's questions at once over the same video at the larger budget
        _attend("attend_questions", 28, 4, 16, 61, 100, 6554, 32),
        # many long answers after a short prefix of uneven heads: the pages dominate
        _attend("attend_pages_64", 28, 4, 64, 1, 4096, 1024, 64, uneven=True),
        # a prompt kept whole: the prefix dominates
        _attend("attend_long_32", 32, 8, 32, 1, 100, 131072, 16),
        # the fp32 layer
        _attend("attend_f32", 8, 8, 8, 3, 200, 128, 16, dtype="f32"),
    ]


def _logu(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        del c["name"]
        if _cost(c) <= most:
            return c


def _draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    h_q, h_kv = rng.choice([(32, 32), (28, 4), (32, 8), (8, 8), (28, 4)])
    page = rng.choice([8, 16, 16, 32, 64, 128, 256])
    batch = _logu(rng, 1, 64)
    new = 1 if rng.random() < 0.6 else _logu(rng, 2, 64)
    kept = _logu(rng, 1, 4096)
    if op == "attend":
        prefix = 0 if rng.random() < 0.1 else _logu(rng, 1, 16384 if dtype == "f32" else 131072)
        return _attend("", h_q, h_kv, batch, new, kept, prefix, page, dtype=dtype, uneven=rng.random() < 0.3)
    more = dict(dtype=dtype, layout=rng.choice(["half", "half", "interleaved"]), rot=rng.choice([32, 64, 96, 128, 128]),
                axes=rng.choice([1, 1, 3]), norm=rng.random() < 0.5, base=rng.choice([1e4, 5e5, 1e6]), first=_logu(rng, 1, 131072))
    if rng.random() < 0.4:
        more.update(scaling=rng.choice(["linear", "ntk", "yarn"]), factor=rng.choice([2.0, 4.0, 8.0]))
    if op == "rotate":
        return _rot("", h_q, h_kv, _logu(rng, 1, 32768), **more)
    return _append("", h_q, h_kv, batch, rng.choice([new, _logu(rng, 2, 512)]), kept, page, **more)


def _ragged(c):
    """(new tokens, tokens in the cache with them) of every sequence: from the case alone."""
    rng = random.Random("%d %d %d" % (c["batch"], c["new"], c["kept"]))
    new = [rng.randint((c["new"] + 1) // 2, c["new"]) for _ in range(c["batch"])]
    kept = [rng.randint(0, c["kept"]) for _ in range(c["batch"])]
    new[0], kept[0] = c["new"], c["kept"]
    return new, [n + k for n, k in zip(new, kept)]


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
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "rotate":
        n = c["tokens"] * (c["h_q"] + c["h_kv"])
        return {"bytes": 2 * n * D * e + c["axes"] * c["tokens"] * 4, "flops": n * (3 * c["rot"] + (4 * D if c["norm"] else 0))}
    new, lens = _ragged(c)
    tokens = sum(new)
    pages = sum(-(-x // c["page"]) for x in lens)
    if c["op"] == "append":
        n = tokens * (c["h_q"] + c["h_kv"])
        return {"bytes": 2 * (n + tokens * c["h_kv"]) * D * e + (c["axes"] + 1) * tokens * 4,
                "flops": n * (3 * c["rot"] + (4 * D if c["norm"] else 0))}
    rows = sum(_prefix_rows(c))
    g = c["h_q"] // c["h_kv"]
    pairs = tokens * g * rows + c["h_q"] * sum(n * x - n * (n - 1) // 2 for n, x in zip(new, lens))
    return {"bytes": 2 * (rows + c["h_kv"] * sum(lens)) * D * e + 2 * tokens * c["h_q"] * D * e + 4 * pages + 8 * c["batch"],
            "flops": 4 * D * pairs}


# ---------------------------------------------------------------- inputs
def _frequencies(c):
    """Radians a position, one for each rotated pair, and the factor of cos and sin."""
    rot, base, s = c["rot"], c["base"], c["factor"]
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if c["scaling"] == "linear":
        return [x / s for x in f], 1.0
    if c["scaling"] == "ntk":
        base = base * s ** (rot / (rot - 2.0))
        return [base ** (-2.0 * i / rot) for i in range(rot // 2)], 1.0
    if c["scaling"] == "yarn":
        edge = lambda turns: rot * math.log(ORIGINAL / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(edge(32.0)), 0), min(math.ceil(edge(1.0)), rot - 1)
        ramp = [min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0) for i in range(rot // 2)]
        return [x / s * r + x * (1 - r) for x, r in zip(f, ramp)], 0.1 * math.log(s) + 1.0
    return f, 1.0


ORIGINAL = 8192  # positions that the scaled frequencies were made for


def _sections(c):
    """Frequencies a position axis turns: all, or a quarter by time and the rest by height and width in equal parts."""
    F = c["rot"] // 2
    return (F,) if c["axes"] == 1 else (F - 2 * (3 * F // 8), 3 * F // 8, 3 * F // 8)


def _positions(c, tokens, starts, g):
    """[axes][tokens]: time runs on from the case's first; height and width lag within a frame of 32 x 40 patches."""
    t = torch.arange(tokens, device=DEV) + c["first"] if starts is None else starts + c["first"]
    if c["axes"] == 1:
        return t[None].int().contiguous()
    return torch.stack([t, t - torch.randint(0, min(32, c["first"] + 1), (tokens,), generator=g, device=DEV),
                        t - torch.randint(0, min(40, c["first"] + 1), (tokens,), generator=g, device=DEV)]).int().contiguous()


def _keys(shape, g, dt):
    """Keys in a narrow cone, shape [..., h_kv, d] with the heads' direction on the last but one axis."""
    u = torch.randn(shape[-2], D, generator=g, device=DEV)
    u = u / torch.linalg.vector_norm(u, dim=1, keepdim=True)
    return u, lambda n: (4.0 * u + torch.randn(*n, shape[-2], D, generator=g, device=DEV)).to(dt)


def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    dt, h_q, h_kv = TYPES[c["dtype"]], c["h_q"], c["h_kv"]
    rnd = lambda *n: torch.randn(*n, generator=g, device=DEV)  # noqa: E731
    s = {"case": c}
    if c["op"] == "rotate":
        tokens, slots = c["tokens"], None
    else:
        new, lens = _ragged(c)
        tokens = sum(new)
        # a pool of pages that the sequences hold in any order, some of it free
        cols = max(-(-x // c["page"]) for x in lens) + 1
        need = [-(-x // c["page"]) for x in lens]
        n_pages = sum(need) + 3
        order = torch.randperm(n_pages, generator=g, device=DEV).int()
        table = torch.zeros(c["batch"], cols, dtype=torch.int32)
        used = torch.cat([torch.zeros(1, dtype=torch.int64), torch.tensor(need).cumsum(0)])
        col = torch.arange(cols)
        inside = col < torch.tensor(need)[:, None]
        table[inside] = (used[:-1, None] + col)[inside].int()
        s["table"] = torch.where(inside.to(DEV), order[table.long().to(DEV)], torch.zeros((), dtype=torch.int32, device=DEV))
        s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["starts"] = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).int().to(DEV)
        s["step"] = c["new"] == 1
        slots = torch.cat([torch.arange(x - n, x) for n, x in zip(new, lens)]).to(DEV)
        u, keys = _keys((h_kv, D), g, dt)
        # [page][head][slot][d]: slots that no sequence has reached hold what was there before
        s["k_pages"] = keys((n_pages, c["page"])).transpose(1, 2).contiguous()
        s["v_pages"] = rnd(n_pages, h_kv, c["page"], D).to(dt)
    if c["op"] == "attend":
        s["q"] = (4.0 * u.repeat_interleave(h_q // h_kv, 0) + rnd(tokens, h_q, D)).to(dt)
        rows = _prefix_rows(c)
        s["prefix_off"] = torch.tensor([0] + rows, dtype=torch.int32).cumsum(0).int().to(DEV)
        if c["uneven"]:
            head = torch.repeat_interleave(torch.arange(h_kv), torch.tensor(rows)).to(DEV)
            s["prefix_k"] = (4.0 * u[head] + rnd(sum(rows), D)).to(dt)
            s["prefix_v"] = rnd(sum(rows), D).to(dt)
        else:
            s["prefix_k"] = keys((rows[0],)).transpose(0, 1).contiguous()
            s["prefix_v"] = rnd(h_kv, rows[0], D).to(dt)
        # what the plain form sees of the batch: places of the tokens and rows in rectangles
        s["batch_max"], s["len_max"], s["row_max"] = max(new), max(lens), max(rows)
        s["out"] = torch.empty(tokens, h_q, D, dtype=dt, device=DEV)
    else:
        # queries, keys and values as one projection gives them: [token][heads of q, k and v][d]
        qkv = rnd(tokens, h_q + 2 * h_kv, D).to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :h_q], qkv[:, h_q:h_q + h_kv], qkv[:, h_q + h_kv:]
        s["pos"] = _positions(c, tokens, slots, g)
        s["q_norm"] = (1.0 + 0.1 * rnd(D)).to(dt) if c["norm"] else None
        s["k_norm"] = (1.0 + 0.1 * rnd(D)).to(dt) if c["norm"] else None
        s["q_out"] = torch.empty(tokens, h_q, D, dtype=dt, device=DEV)
        # a prompt's keys go where the eviction pass reads them: [head][token][d]
        s["k_out"] = torch.empty(h_kv, tokens, D, dtype=dt, device=DEV).transpose(0, 1)
        # the plain form's tables of cos and sin, made once in 64 bits as a model makes them
        freq, mag = _frequencies(c)
        last = c["first"] + (tokens if slots is None else c["new"] + c["kept"]) + 1
        turn = torch.arange(last, dtype=torch.float64, device=DEV)[:, None] * torch.tensor(freq, dtype=torch.float64, device=DEV)
        s["cos"], s["sin"] = (mag * turn.cos()).float(), (mag * turn.sin()).float()
        s["axis"] = torch.repeat_interleave(torch.arange(c["axes"]), torch.tensor(_sections(c))).to(DEV)
    if own:  # the handles and the workspace that a program keeps for a model and its cache
        from paper_2609_06663_gb300 import ecokv as E
        if c["op"] == "attend":
            s["prefix"] = E.Prefix(s["prefix_k"], s["prefix_v"], s["prefix_off"] if c["uneven"] else None)
            s["ws"] = E.alloc_attend_workspace(tokens, c["batch"], h_q, h_kv, dt)
        else:
            s["rotary"] = E.rotary(c["rot"], c["base"], layout=c["layout"], scaling=c["scaling"], factor=c["factor"],
                                   original=ORIGINAL, sections=_sections(c))
        if c["op"] != "rotate":
            s["cache"] = E.PagedCache(s["k_pages"], s["v_pages"], s["table"], s["lengths"])
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    return (_run_own if own else _run_plain)[s["case"]["op"]](s)


def _own_rotate(s):
    from paper_2609_06663_gb300 import ecokv as E
    return E.rotate(s["rotary"], s["pos"], s["q"], s["k"], q_norm=s["q_norm"], k_norm=s["k_norm"], q_out=s["q_out"],
                    k_out=s["k_out"])


def _own_append(s):
    from paper_2609_06663_gb300 import ecokv as E
    q = E.append(s["cache"], s["k"], s["v"], starts=None if s["step"] else s["starts"], rotary=s["rotary"],
                 positions=s["pos"], q=s["q"], q_norm=s["q_norm"], k_norm=s["k_norm"], q_out=s["q_out"])
    return q, s["k_pages"], s["v_pages"]


def _own_attend(s):
    from paper_2609_06663_gb300 import ecokv as E
    return E.attend(s["q"], s["prefix"], s["cache"], starts=None if s["step"] else s["starts"], out=s["out"], ws=s["ws"])


def _turned(s, x, w):
    """Norm and rotation of x [tokens, heads, D] in 32 bits."""
    c = s["case"]
    x, rot, F = x.float(), c["rot"], c["rot"] // 2
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
    place = s["pos"].long()[s["axis"]]  # [F, tokens]
    f = torch.arange(F, device=DEV)[:, None]
    cos, sin = s["cos"][place, f].t()[:, None], s["sin"][place, f].t()[:, None]
    if c["layout"] == "half":
        a, b = x[..., :F], x[..., F:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_rotate(s):
    return tuple(_turned(s, s[n], s[n + "_norm"]).to(s["q"].dtype) for n in ("q", "k"))


def _places(s):
    """(sequence, slot) of every new token."""
    starts, lengths = s["starts"].long(), s["lengths"].long()
    t = torch.arange(s["q"].shape[0], device=DEV)
    b = torch.searchsorted(starts, t, right=True) - 1
    return b, lengths[b] - starts[b + 1] + t


def _plain_append(s):
    page, dt = s["case"]["page"], s["q"].dtype
    b, slot = _places(s)
    at = s["table"].long()[b, slot // page]
    s["k_pages"][at, :, slot % page] = _turned(s, s["k"], s["k_norm"]).to(dt)
    s["v_pages"][at, :, slot % page] = s["v"]
    return _turned(s, s["q"], s["q_norm"]).to(dt), s["k_pages"], s["v_pages"]


def _plain_attend(s):
    c = s["case"]
    q, h_q, h_kv, page = s["q"], c["h_q"], c["h_kv"], c["page"]
    tokens, g, B, T, L, P = q.shape[0], h_q // h_kv, c["batch"], s["batch_max"], s["len_max"], s["row_max"]
    scale = 1.0 / math.sqrt(D)
    ninf = torch.full((), float("-inf"), device=DEV)
    qf = q.float().view(tokens, h_kv, g, D) * scale
    pk, pv = s["prefix_k"], s["prefix_v"]
    off = s["prefix_off"].long()
    if c["uneven"]:  # the heads' rows as a rectangle
        at = off[:-1, None] + torch.arange(P, device=DEV)
        live = at < off[1:, None]
        at = at.clamp(max=pk.shape[0] - 1)
        pk, pv = pk[at], pv[at] * live[..., None]
    # scores of the prefix: [h_kv, tokens * g, P]
    qh = qf.transpose(0, 1).reshape(h_kv, tokens * g, D)
    sp = qh @ pk.float().transpose(1, 2)
    if c["uneven"]:
        sp = torch.where(live[:, None], sp, ninf)
    sp = sp.view(h_kv, tokens, g, P)
    # the batch's own keys as a rectangle [B, h_kv, L, D], its queries as [B, h_kv, T * g, D]
    b, slot = _places(s)
    i = torch.arange(tokens, device=DEV) - s["starts"].long()[b]
    cols = -(-L // page)
    own_k, own_v = (x[s["table"][:, :cols].long()].transpose(1, 2).reshape(B, h_kv, cols * page, D)[:, :, :L].float()
                    for x in (s["k_pages"], s["v_pages"]))
    qb = torch.zeros(B, T, h_kv, g, D, device=DEV)
    qb[b, i] = qf
    so = qb.permute(0, 2, 1, 3, 4).reshape(B, h_kv, T * g, D) @ own_k.transpose(2, 3)
    so = so.view(B, h_kv, T, g, L)[b, :, i].transpose(0, 1)  # [h_kv, tokens, g, L]
    so = torch.where(torch.arange(L, device=DEV) <= slot[:, None, None], so, ninf)
    top = so.amax(-1, keepdim=True)
    if P:
        top = torch.maximum(top, sp.amax(-1, keepdim=True))
    ep, eo = torch.exp(sp - top), torch.exp(so - top)
    total = ep.sum(-1, keepdim=True) + eo.sum(-1, keepdim=True)
    out = (ep.view(h_kv, tokens * g, P) @ pv.float()).view(h_kv, tokens, g, D)
    eb = torch.zeros(B, T, h_kv, g, L, device=DEV)
    eb[b, i] = eo.transpose(0, 1)
    ob = eb.permute(0, 2, 1, 3, 4).reshape(B, h_kv, T * g, L) @ torch.where(
        (torch.arange(L, device=DEV) < s["lengths"][:, None])[:, None, :, None], own_v, torch.zeros((), device=DEV))
    out = out + ob.view(B, h_kv, T, g, D)[b, :, i].transpose(0, 1)
    return (out / total).transpose(0, 1).reshape(tokens, h_q, D).to(q.dtype)


_run_own = {"rotate": _own_rotate, "append": _own_append, "attend": _own_attend}
_run_plain = {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend}


# ---------------------------------------------------------------- from the definitions, in 64 bits
def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "attend":
        return _exact_attend(c, s)
    freq, mag = _frequencies(c)
    pos = s["pos"].double()
    turn = torch.stack([pos[a] * f for f, a in zip(freq, s["axis"].tolist())], -1)  # [tokens, F]
    unit = torch.polar(torch.full_like(turn, mag), turn)[:, None]
    done = []
    for x, w in ((s["q"], s["q_norm"]), (s["k"], s["k_norm"])):
        x = x.double()
        if w is not None:
            x = x / (x.square().sum(-1, keepdim=True) / D + 1e-6).sqrt() * w.double()
        z = x[..., :c["rot"]]
        z = z.unflatten(-1, (2, -1)).transpose(-1, -2) if c["layout"] == "half" else z.unflatten(-1, (-1, 2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * unit)
        z = z.transpose(-1, -2).flatten(-2) if c["layout"] == "half" else z.flatten(-2)
        done.append(torch.cat([z, x[..., c["rot"]:]], -1))
    if c["op"] == "rotate":
        return tuple(done)
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    new, lens = _ragged(c)
    t = 0
    for b, (n, x) in enumerate(zip(new, lens)):
        slot = torch.arange(x - n, x, device=DEV)
        at = s["table"][b, slot // c["page"]].long()
        kp[at, :, slot % c["page"]] = done[1][t:t + n]
        vp[at, :, slot % c["page"]] = s["v"][t:t + n].double()
        t += n
    return done[0], kp, vp


def _exact_attend(c, s):
    new, lens = _ragged(c)
    off = [0]
    for n in _prefix_rows(c):
        off.append(off[-1] + n)
    g, t, out = c["h_q"] // c["h_kv"], 0, torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    if work(c)["flops"] > 3e12:
        return None
    pk, pv = s["prefix_k"].reshape(-1, D), s["prefix_v"].reshape(-1, D)
    for h in range(c["h_kv"]):  # a head's prefix in 64 bits, then each sequence
        hk, hv = pk[off[h]:off[h + 1]].double(), pv[off[h]:off[h + 1]].double()
        t = 0
        for b, (n, x) in enumerate(zip(new, lens)):
            ids = s["table"][b, :-(-x // c["page"])].long()
            k = torch.cat([hk, s["k_pages"][ids, h].reshape(-1, D)[:x].double()])
            v = torch.cat([hv, s["v_pages"][ids, h].reshape(-1, D)[:x].double()])
            q = s["q"][t:t + n, h * g:(h + 1) * g].double()
            score = torch.einsum("ngd,kd->ngk", q, k) * D ** -0.5
            seen = torch.arange(k.shape[0], device=DEV) - hk.shape[0] <= torch.arange(x - n, x, device=DEV)[:, None]
            p = torch.softmax(score.masked_fill(~seen[:, None], float("-inf")), -1)
            out[t:t + n, h * g:(h + 1) * g] = torch.einsum("ngk,kd->ngd", p, v)
            t += n
    return out
