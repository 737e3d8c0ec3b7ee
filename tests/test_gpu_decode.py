"""The decode step's operators against their definitions in 64 bits.

Tolerances.  u = 2^-24, w = 2^-8 (bf16's rounding) or 0 for fp32.

Rotation: the angle is rounded once to 24 bits of a half turn (pi u of an angle),
sine and cosine are good to 2 ulp, then a factor, two products and a sum, and with a
norm a mean of 128 squares, a root and two products: 16 u of |x_a| + |x_b| covers
them (24 u with a norm), and w |y| the result's rounding.

Attention: a score is a sum of 128 products, off by at most 128 u of sum |q||k| scale
(call it mag) and a few u for the scale and the subtraction of the maximum, the
exponential by 2^-21; a weight is then off by d = (140 mag + 40) u relative, and a
quotient of sums by 2 d and the sums' own roundings, (keys + 300) u.  For bf16
each weight is rounded once (w) and the result too.
"""
import math

import pytest
import torch

from paper_2609_06663_gb300 import ecokv as E
from tests.decode_ref import attend as ref_attend
from tests.decode_ref import frequencies, turn

pytestmark = pytest.mark.gpu
U, D = 2.0 ** -24, 128
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
W = {"bf16": 2.0 ** -8, "f32": 0.0}


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


# ---------------------------------------------------------------- rotate
ROTATE = [  # tokens, h_q, h_kv, layout, rot, sections, norm, scaling, first
    (1, 4, 2, "half", 128, None, False, "none", 0),
    (1, 32, 8, "interleaved", 64, None, True, "none", 7),
    (33, 28, 4, "half", 128, (16, 24, 24), False, "none", 131000),
    (7, 3, 1, "half", 96, (5, 20, 23), True, "yarn", 70000),
    (130, 8, 8, "interleaved", 128, (63, 1), False, "linear", 2 ** 31 - 200),
    (513, 2, 2, "half", 16, (2, 2, 2, 2), True, "ntk", -300),
    (4097, 5, 1, "half", 32, None, False, "none", 0),
    (64, 28, 4, "interleaved", 112, None, True, "yarn", 1000000),
]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,h_q,h_kv,layout,rot,sections,norm,scaling,first", ROTATE)
def test_rotate(tokens, h_q, h_kv, layout, rot, sections, norm, scaling, first, dt):
    g = gen(tokens + rot)
    T = TYPES[dt]
    r = E.rotary(rot, 1e4, layout, scaling, 4.0, 8192, sections)
    freq, mag = frequencies(rot, 1e4, scaling, 4.0, 8192)
    qkv = (3 * torch.randn(tokens, h_q + 2 * h_kv, D, generator=g)).to(T)
    pos = torch.stack([torch.arange(first, first + tokens) - (3 * x if first >= 0 else 0) for x in range(r.axes)]).int()
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(T) if norm else None for _ in range(2)]
    dev = qkv.cuda()
    q, k = dev[:, :h_q], dev[:, h_q:h_q + h_kv]
    k_out = torch.full((h_kv, tokens + 2, D), 7.0, dtype=T, device="cuda")
    qo, ko = E.rotate(r, pos.cuda(), q, k, *[None if x is None else x.cuda() for x in w], eps=1e-5,
                      k_out=k_out[:, 1:-1].transpose(0, 1))
    axis = list(r.axis)
    for got, x, n in ((qo, qkv[:, :h_q], w[0]), (ko, qkv[:, h_q:h_q + h_kv], w[1])):
        want, size = turn(x, pos, freq, axis, layout, mag, n, 1e-5)
        tol = (24 if norm else 16) * U * size + W[dt] * want.abs() * (1 + 2 ** -7) + 1e-30
        if not norm:
            tol[..., rot:] = 0.0  # copied
        assert bool(((got.cpu().double() - want).abs() <= tol).all())
    assert bool((k_out[:, 0] == 7).all()) and bool((k_out[:, -1] == 7).all())
    assert torch.equal(dev.cpu(), qkv)
    # in place, and the norms alone
    qi = q.clone(memory_format=torch.contiguous_format)
    assert E.rotate(r, pos.cuda(), qi, q_norm=None if w[0] is None else w[0].cuda(), eps=1e-5, q_out=qi)[0] is qi
    assert torch.equal(qi, qo)
    if norm:
        alone = E.rotate(None, None, q, q_norm=w[0].cuda(), eps=1e-5)[0]
        want, size = turn(qkv[:, :h_q], None, None, None, layout, norm=w[0], eps=1e-5)
        assert bool(((alone.cpu().double() - want).abs() <= 24 * U * size + W[dt] * want.abs() * (1 + 2 ** -7)).all())


def test_rotation_undoes_itself_and_keeps_lengths():
    # the angles of p and -p cancel, whatever the position: two rotations' roundings are left
    g = gen(3)
    r = E.rotary(128, 1e6)
    x = torch.randn(1000, 4, D, generator=g).cuda()
    pos = torch.randint(-2 ** 31 + 1, 2 ** 31 - 1, (1, 1000), generator=g).int().cuda()
    y = E.rotate(r, pos, x)[0]
    z = E.rotate(r, -pos, y)[0]
    size = (x[..., :64].abs() + x[..., 64:].abs()).repeat(1, 1, 2)
    assert bool(((z - x).abs() <= 64 * U * size).all())
    assert bool(((y.double().norm(dim=-1) / x.double().norm(dim=-1) - 1).abs() <= 32 * U).all())


# ---------------------------------------------------------------- the paged cache
class Batch:
    """Ragged sequences with their pages in any order; free slots hold NaN."""

    def __init__(self, seed, h_kv, new, lens, page, dt, order="head", spare=3, cols=None):
        g = gen(seed)
        T = TYPES[dt]
        self.new, self.lens, self.page, self.h_kv = new, lens, page, h_kv
        need = [-(-x // page) for x in lens]
        cols = cols or max(need + [1]) + 1
        n = sum(need) + spare
        shape = {"head": (n, h_kv, page, D), "slot": (n, page, h_kv, D)}[order]
        self.k, self.v = (torch.full(shape, math.nan, dtype=T) for _ in range(2))
        if order == "slot":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        perm = torch.randperm(n, generator=g).tolist()
        self.table = torch.full((len(lens), cols), 2 ** 30, dtype=torch.int32)  # not to be read past a sequence's pages
        self.own = []
        for b, x in enumerate(lens):
            ok, ov = torch.randn(2, h_kv, x, D, generator=g).to(T)
            for c in range(need[b]):
                p = perm.pop()
                self.table[b, c] = p
                m = min(page, x - c * page)
                self.k[p, :, :m] = ok[:, c * page:c * page + m]
                self.v[p, :, :m] = ov[:, c * page:c * page + m]
            self.own.append((ok, ov))
        self.starts = torch.tensor([0] + new).cumsum(0).int()
        self.tokens = sum(new)
        self.free = perm
        # (to the device with the same strides)
        self.dk, self.dv = (x.cuda() if order == "head" else x.transpose(1, 2).cuda().transpose(1, 2) for x in (self.k, self.v))
        self.cache = E.PagedCache(self.dk, self.dv, self.table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())


APPEND = [  # h_q, h_kv, new, lengths with them, page, order, norm, sections
    (4, 2, [1], [1], 8, "head", False, None),
    (28, 4, [1] * 5, [1, 17, 16, 300, 33], 16, "slot", False, (16, 24, 24)),
    (8, 8, [3, 0, 70, 1, 9], [3, 5, 200, 64, 65], 32, "head", True, None),
    (32, 8, [0, 40, 40], [0, 41, 1000], 512, "slot", True, None),
    (2, 1, [1] * 70, list(range(1, 71)), 8, "head", False, None),
]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("h_q,h_kv,new,lens,page,order,norm,sections", APPEND)
def test_append(h_q, h_kv, new, lens, page, order, norm, sections, dt):
    b = Batch(1, h_kv, new, lens, page, dt, order)
    g, T = gen(2), TYPES[dt]
    r = E.rotary(128, 1e6, sections=sections)
    freq, mag = frequencies(128, 1e6)
    qkv = torch.randn(b.tokens, h_q + 2 * h_kv, D, generator=g).to(T)
    pos = torch.randint(0, 200000, (r.axes, b.tokens), generator=g).int()
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(T).cuda() if norm else None for _ in range(2)]
    dev = qkv.cuda()
    q, k, v = dev[:, :h_q], dev[:, h_q:h_q + h_kv], dev[:, h_q + h_kv:]
    one = all(n == 1 for n in new)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    qo = E.append(b.cache, k, v, None if one else b.starts.cuda(), r, pos.cuda(), q, w[0], w[1], ws=ws)
    # the rows are the ones that rotate() gives
    q2, k2 = E.rotate(r, pos.cuda(), q, k, w[0], w[1])
    assert torch.equal(qo, q2)
    want_k, want_v, t = b.k.clone(), b.v.clone(), 0
    for s, (n, x) in enumerate(zip(new, lens)):
        for slot in range(x - n, x):
            p = int(b.table[s, slot // page])
            want_k[p, :, slot % page] = k2[t].cpu()
            want_v[p, :, slot % page] = qkv[t, h_q + h_kv:]
            t += 1
    for got, want in ((b.dk.cpu(), want_k), (b.dv.cpu(), want_v)):
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())
    want, size = turn(qkv[:, h_q:h_q + h_kv], pos, freq, list(r.axis), "half", mag, None if w[1] is None else w[1].cpu())
    assert bool(((k2.cpu().double() - want).abs() <= 24 * U * size + W[dt] * want.abs() * (1 + 2 ** -7) + 1e-30).all())
    assert E.ecokv_device_status(ws) == 0
    # without rotation and without queries: copies
    if not norm:
        E.append(b.cache, k, v, None if one else b.starts.cuda())
        p, s = int(b.table[0, (lens[0] - 1) // page]), (lens[0] - 1) % page
        assert torch.equal(b.dk[p, :, s], k[new[0] - 1]) and torch.equal(b.dv[p, :, s], v[new[0] - 1])


def test_append_skips_what_has_no_slot_and_says_so():
    b = Batch(5, 2, [2, 1, 1, 1], [20, 5, 9, 3], 8, "f32", cols=3)
    before = b.dk.clone(), b.dv.clone()
    k, v = torch.randn(2, 5, 2, D, device="cuda")
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    b.cache.table[1, 0] = 10 ** 6      # a page that is not there
    b.cache.table[2, 1] = -1
    b.cache.lengths[3] = 25            # past the table's columns
    b.cache.lengths[0] = 1             # two new tokens in one slot: the first has none
    E.append(b.cache, k, v, b.starts.cuda(), ws=ws)
    assert E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX
    assert E.ecokv_device_status(ws) == 0
    p = int(b.table[0, 0])
    for got, was, new in ((b.dk, before[0], k), (b.dv, before[1], v)):
        assert torch.equal(got[p, :, 0], new[1])
        got[p, :, 0] = was[p, :, 0]
        assert torch.equal(got.nan_to_num(), was.nan_to_num())


# ---------------------------------------------------------------- attention
def make_prefix(g, rows, dt, uneven):
    """rows of every head -> (per head (k, v), E.Prefix)"""
    T = TYPES[dt]
    heads = [tuple(torch.randn(2, n, D, generator=g).to(T)) for n in rows]
    if uneven:
        off = torch.tensor([0] + rows).cumsum(0).int().cuda()
        return heads, E.Prefix(*(torch.cat([h[i] for h in heads]).cuda() for i in range(2)), off)
    # the layer's rows with room between the heads, as a layered budget leaves them
    k, v = (torch.full((len(rows), rows[0] + 3, D), math.nan, dtype=T) for _ in range(2))
    for h, (hk, hv) in enumerate(heads):
        k[h, :rows[0]], v[h, :rows[0]] = hk, hv
    return heads, E.Prefix(k.cuda()[:, :rows[0]], v.cuda()[:, :rows[0]])


def check_attend(b, heads, pre, h_q, dt, q=None, flags=0, scale=0.0, seed=9, **kw):
    T = TYPES[dt]
    if q is None:
        q = (2 * torch.randn(b.tokens, h_q, D, generator=gen(seed))).to(T)
    one = all(n == 1 for n in b.new)
    lse = torch.full((b.tokens, h_q), 5.0, device="cuda")
    ws = E.alloc_attend_workspace(b.tokens, len(b.new), h_q, b.h_kv, T)
    ws[256:].fill_(255)  # what a call does not write it must not read
    out = E.attend(q.cuda(), pre, b.cache, None if one else b.starts.cuda(), lse=lse, flags=flags, ws=ws, scale=scale, **kw)
    assert E.ecokv_device_status(ws) == 0
    sc = scale or 1 / math.sqrt(D)
    want, size, wl, mag = ref_attend(q, heads, b.own, b.new, sc)
    d = (140 * mag + 40) * U
    keys = max([len(h[0]) for h in heads] + [0]) + max(b.lens)
    tol = (2 * d + (keys + 300) * U + W[dt]) * size + W[dt] * want.abs() * (1 + 2 ** -7)
    got = out.cpu().double()
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() - tol).max())
    empty = wl == -math.inf
    assert torch.equal(lse.cpu() == -math.inf, empty) and bool((got[empty] == 0).all())
    assert bool(((lse.cpu().double() - wl)[~empty].abs() <= d + (keys + 300) * U + 4 * U * wl[~empty].abs()).all())
    again = E.attend(q.cuda(), pre, b.cache, None if one else b.starts.cuda(), flags=flags, ws=ws, scale=scale, **kw)
    assert torch.equal(again, out)  # the same bits every time
    return out


ATTEND = [  # h_q, h_kv, new, lengths, page, prefix rows (a list: uneven), order
    (4, 4, [1], [1], 16, 0, "head"),                                        # one key
    (4, 2, [1, 1], [5, 130], 8, 1, "head"),
    (28, 4, [1] * 5, [1, 16, 17, 128, 129], 16, 127, "slot"),
    (28, 4, [1] * 9, [3, 1, 700, 5, 64, 63, 65, 2, 256], 32, 129, "head"),
    (32, 8, [1] * 40, [1 + 7 * i for i in range(40)], 64, 385, "slot"),     # 160 rows a head: two row tiles
    (8, 8, [3, 0, 5, 1], [3, 0, 200, 640], 16, 128, "head"),
    (28, 4, [61, 30, 1, 17, 33], [61, 100, 1, 400, 33], 128, 260, "head"),  # questions
    (8, 1, [150], [300], 512, 40, "slot"),                                  # many token groups of one sequence
    (64, 1, [1, 2, 5], [9, 20, 500], 256, 64, "head"),                      # the largest group
    (6, 2, [2, 2, 2, 2], [1, 0, 2, 30], 16, 0, "head"),                     # tokens that see nothing
    (6, 2, [1, 1, 1], [0, 0, 0], 8, 0, "head"),                             # none that sees anything
    (10, 5, [1] * 33, [2] * 33, 8, [0, 300, 1, 128, 77], "head"),           # uneven heads, one of them empty
    (12, 4, [4, 9], [40, 1000], 16, [1000, 0, 0, 513], "slot"),
    (40, 40, [1] * 3, [40, 50, 600], 16, [i % 7 * 40 for i in range(40)], "head"),  # more heads than lanes
]


@pytest.mark.parametrize("dt,flags", [("bf16", 0), ("bf16", E.ECOKV_FLAG_FORCE_SIMT), ("f32", 0)])
@pytest.mark.parametrize("h_q,h_kv,new,lens,page,prefix,order", ATTEND)
def test_attend(h_q, h_kv, new, lens, page, prefix, order, dt, flags):
    # (a length below the new tokens: those in front have no slot and see the prefix alone)
    b = Batch(11, h_kv, new, lens, page, dt, order)
    rows = prefix if isinstance(prefix, list) else [prefix] * h_kv
    heads, pre = make_prefix(gen(4), rows, dt, isinstance(prefix, list))
    check_attend(b, heads, pre if sum(rows) else None, h_q, dt, flags=flags)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attend_prefix_alone_and_strides(dt):
    g = gen(21)
    heads, pre = make_prefix(g, [200] * 4, dt, False)
    b = Batch(1, 4, [1] * 20, [0] * 20, 16, dt)
    q = torch.randn(20, 8, D, generator=g).to(TYPES[dt])
    want = check_attend(b, heads, pre, 8, dt, q=q)
    # no cache at all; queries from a wider projection, the output in another order
    wide = torch.zeros(20, 11, D, dtype=TYPES[dt], device="cuda")
    wide[:, 2:10] = q.cuda()
    out = torch.full((8, 22, D), 3.0, dtype=TYPES[dt], device="cuda")
    got = E.attend(wide[:, 2:10], pre, None, out=out[:, 1:21].transpose(0, 1))
    assert torch.equal(got, want) and bool((out[:, 0] == 3).all()) and bool((out[:, 21] == 3).all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attend_large_scores_and_growing_maxima(dt):
    """Scores that grow along the keys by far more than an exponential's range, in the prefix, the pages and between them."""
    g = gen(31)
    h_kv, n = 2, 700
    b = Batch(3, h_kv, [2, 1], [400, 333], 16, dt)
    u = torch.randn(D, generator=g)
    u /= u.norm()
    T = TYPES[dt]
    ramp = torch.linspace(-30, 30, n)[:, None]
    heads = [((ramp * u * s + 0.1 * torch.randn(n, D, generator=g)).to(T), torch.randn(n, D, generator=g).to(T))
             for s in (1, -1)]
    pre = E.Prefix(*(torch.stack([h[i] for h in heads]).cuda() for i in range(2)))
    q = (100 * u * torch.tensor([1.0, -1.0, 0.3, 2.0])[None, :, None] + torch.zeros(3, 4, D)).to(T)
    check_attend(b, heads, pre, 4, dt, q=q)
    check_attend(b, heads, pre, 4, dt, q=q, scale=1.5)


def test_attend_pages_past_32_bit_offsets():
    """Pages beyond 2^32 elements of the pool."""
    h_kv, page = 8, 4096
    n_pages = 2 ** 32 // (h_kv * page * D) + 3
    k = torch.empty(n_pages, h_kv, page, D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    g = gen(41)
    L = page + 5
    ok, ov = torch.randn(2, h_kv, L, D, generator=g).bfloat16()
    ids = [n_pages - 1, n_pages - 2]
    for c, p in enumerate(ids):
        m = min(page, L - c * page)
        k[p, :, :m], v[p, :, :m] = ok[:, c * page:c * page + m].cuda(), ov[:, c * page:c * page + m].cuda()
    b = Batch(1, h_kv, [1], [1], 8, "bf16")
    b.lens, b.own = [L], [(ok, ov)]
    b.cache = E.PagedCache(k, v, torch.tensor([ids], dtype=torch.int32).cuda(), torch.tensor([L], dtype=torch.int32).cuda())
    none = [(torch.zeros(0, D), torch.zeros(0, D))] * h_kv
    check_attend(b, none, None, 16, "bf16")
    check_attend(b, none, None, 16, "bf16", flags=E.ECOKV_FLAG_FORCE_SIMT)
    kn, vn = torch.randn(2, 1, h_kv, D, generator=g).bfloat16()
    E.append(b.cache, kn.cuda(), vn.cuda())
    assert torch.equal(k[ids[1], :, 4].cpu(), kn[0]) and torch.equal(v[ids[1], :, 4].cpu(), vn[0])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attend_reports_bad_device_data(dt):
    b = Batch(6, 2, [1] * 3, [40, 20, 30], 16, dt)
    q = torch.randn(3, 4, D, generator=gen(1)).to(TYPES[dt]).cuda()
    ws = E.alloc_attend_workspace(3, 3, 4, 2, q.dtype)
    good = E.attend(q, None, b.cache, ws=ws)
    assert E.ecokv_device_status(ws) == 0
    for what in ("page", "negative", "length", "starts", "head_off"):
        table, lengths, starts, pre = b.table.clone().cuda(), torch.tensor(b.lens).int().cuda(), None, None
        if what == "page":
            table[1, 0] = 2 ** 30
        if what == "negative":
            table[1, 1] = -5
        if what == "length":
            lengths[1] = 10 ** 6
        if what == "starts":
            starts = torch.tensor([0, 1, 0, 3]).int().cuda()
        if what == "head_off":
            pre = E.Prefix(*(torch.zeros(10, D, dtype=q.dtype, device="cuda") for _ in range(2)),
                           torch.tensor([0, 50, 10]).int().cuda())
        if what == "length":  # every column of the table is a page that is there
            table[table == 2 ** 30] = 0
        out = E.attend(q, pre, E.PagedCache(b.dk.nan_to_num(), b.dv.nan_to_num(), table, lengths), starts, ws=ws)
        assert E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX, what
        if what in ("page", "negative", "length"):
            assert torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])
    assert torch.equal(E.attend(q, None, b.cache, ws=ws), good)


def test_attend_refuses_what_does_not_fit():
    b = Batch(1, 2, [1] * 3, [4, 5, 6], 8, "bf16")
    q = torch.zeros(3, 4, D, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        E.attend(q.float(), None, b.cache)
    with pytest.raises(ValueError):
        E.attend(q, None, None)
    with pytest.raises(ValueError):
        E.attend(q[:, :, :64], None, b.cache)
    with pytest.raises(ValueError):
        E.attend(q, E.Prefix(*(torch.zeros(3, 5, D, dtype=q.dtype, device="cuda") for _ in range(2))), b.cache)
    with pytest.raises(ValueError):
        E.attend(q, None, b.cache, torch.tensor([0, 1, 3], device="cuda").int())
    with pytest.raises(ValueError):
        E.attend(q, None, b.cache, torch.tensor([0, 1, 2, 3], device="cuda"))
    with pytest.raises(ValueError):
        E.append(b.cache, q, q)
    with pytest.raises(E.EcokvError) as e:
        E.attend(q, None, b.cache, ws=torch.zeros(1024, dtype=torch.uint8, device="cuda"))
    assert e.value.code == E.ECOKV_ERR_WORKSPACE
    with pytest.raises(E.EcokvError):
        E.attend(q[:2], None, b.cache)  # two tokens of three sequences, and no starts


def test_a_decode_step_in_a_graph_on_another_stream():
    """append and attend captured once and replayed as lengths, positions and inputs change."""
    h_q, h_kv, B = 28, 4, 6
    b = Batch(8, h_kv, [1] * B, [30, 1, 15, 16, 100, 63], 16, "bf16", spare=10, cols=10)
    heads, pre = make_prefix(gen(2), [333] * h_kv, "bf16", False)
    r = E.rotary(128, 1e6)
    s = torch.cuda.Stream()
    qkv = torch.zeros(B, h_q + 2 * h_kv, D, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(1, B, dtype=torch.int32, device="cuda")
    q_out, out = (torch.zeros(B, h_q, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = E.alloc_attend_workspace(B, B, h_q, h_kv, torch.bfloat16)
    table = b.table.clone()
    for i in range(B):  # a page for the slots to come
        table[i, -(-b.lens[i] // 16)] = b.free.pop()
    b.cache.table.copy_(table)
    x = [torch.randn(qkv.shape, generator=gen(50 + i)).bfloat16() for i in range(4)]

    def step():
        E.append(b.cache, qkv[:, h_q:h_q + h_kv], qkv[:, h_q + h_kv:], None, r, pos, qkv[:, :h_q], q_out=q_out, ws=ws)
        E.attend(q_out, pre, b.cache, out=out, ws=ws)

    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        step()  # (writes the last slots; what they hold goes back below)
        with torch.cuda.graph(graph, stream=s):
            step()
    torch.cuda.synchronize()
    b.dk.copy_(b.k)
    b.dv.copy_(b.v)
    for i in range(4):
        qkv.copy_(x[i])
        pos.fill_(5000 + i)
        b.cache.lengths += 1
        graph.replay()
        torch.cuda.synchronize()
        k2 = E.rotate(r, pos, qkv[:, :h_q], qkv[:, h_q:h_q + h_kv])
        assert torch.equal(k2[0], q_out)
        b.own = [(torch.cat([ok, k2[1][j].cpu()[:, None]], 1), torch.cat([ov, x[i][j, h_q + h_kv:][:, None]], 1))
                 for j, (ok, ov) in enumerate(b.own)]
        b.lens = [n + 1 for n in b.lens]
        assert torch.equal(check_attend(b, heads, pre, h_q, "bf16", q=q_out.cpu()), out)


def test_attend_waits_that_run_out():
    """The injected stall: a status, an untouched context, and the next call as ever."""
    b = Batch(6, 4, [1] * 3, [40, 200, 300], 16, "bf16")
    heads, pre = make_prefix(gen(2), [500] * 4, "bf16", False)
    q = torch.randn(3, 28, D, generator=gen(1)).bfloat16().cuda()
    ws = E.alloc_attend_workspace(3, 3, 28, 4, q.dtype)
    good = E.attend(q, pre, b.cache, ws=ws)
    E.attend(q, pre, b.cache, ws=ws, flags=E.ECOKV_FLAG_TEST_STALL, timeout_us=20000)
    assert E.ecokv_device_status(ws) == E.ECOKV_ERR_TIMEOUT
    assert torch.equal(E.attend(q, pre, b.cache, ws=ws), good) and E.ecokv_device_status(ws) == 0
    with pytest.raises(E.EcokvError) as e:
        E.attend(q, pre, b.cache, flags=E.ECOKV_FLAG_TEST_STALL | E.ECOKV_FLAG_FORCE_SIMT)
    assert e.value.code == E.ECOKV_ERR_UNSUPPORTED


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("seed", range(6))
def test_attend_random_batches(seed, dt):
    """Batches of up to 70 sequences with and without tokens, slots and prefix rows, any group, page size and order."""
    import random
    r = random.Random(seed)
    h_kv, group = r.choice([1, 2, 3]), r.choice([1, 2, 5, 7, 16, 33])
    one = r.random() < 0.4
    n = r.choice([1, 5, 31, 32, 33, 70])
    new = [1 if one else r.choice([0, 1, 1, 2, r.randint(0, 40)]) for _ in range(n)]
    if sum(new) == 0:
        new[-1] = 3
    lens = [max(0, x + r.choice([-1, 0, 0, 1, 17, r.randint(0, 300)])) for x in new]
    uneven = r.random() < 0.5
    rows = [r.randint(0, 400) for _ in range(h_kv)] if uneven else [r.choice([0, 1, 64, 300])] * h_kv
    b = Batch(seed, h_kv, new, lens, r.choice([8, 16, 64, 256]), dt, r.choice(["head", "slot"]))
    heads, pre = make_prefix(gen(seed), rows, dt, uneven)
    check_attend(b, heads, pre if sum(rows) else None, h_kv * group, dt)


def test_attend_layouts():
    """Queries and outputs by head, K and V side by side in one tensor: the same bits as in their usual order."""
    b = Batch(17, 4, [2, 1, 3], [70, 1, 200], 16, "bf16")
    heads, pre = make_prefix(gen(3), [150] * 4, "bf16", False)
    q = torch.randn(6, 8, D, generator=gen(2)).bfloat16()
    want = check_attend(b, heads, pre, 8, "bf16", q=q)
    both = torch.stack([b.dk, b.dv], 1)          # [pages, 2, heads, slots, d]
    cache = E.PagedCache(both[:, 0], both[:, 1], b.cache.table, b.cache.lengths)
    pkv = torch.stack([pre.k, pre.v], 2)         # [heads, rows, 2, d]
    by_head = q.transpose(0, 1).contiguous().cuda().transpose(0, 1)
    out = torch.zeros(8, 6, D, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    got = E.attend(by_head, E.Prefix(pkv[:, :, 0], pkv[:, :, 1]), cache, b.starts.cuda(), out=out)
    assert got is out and torch.equal(out, want)
    # appended through the other layout
    k, v = torch.randn(2, 6, 4, D, generator=gen(5)).bfloat16().cuda()
    E.append(cache, k, v, b.starts.cuda())
    E.append(b.cache, k, v, b.starts.cuda())
    assert torch.equal(both[:, 0].nan_to_num(), b.dk.nan_to_num()) and torch.equal(both[:, 1].nan_to_num(), b.dv.nan_to_num())


def test_calls_on_two_streams_with_workspaces_of_their_own():
    b = Batch(19, 4, [1] * 9, [50 * i + 1 for i in range(9)], 16, "bf16")
    _, pre = make_prefix(gen(3), [900] * 4, "bf16", False)
    q = [torch.randn(9, 28, D, generator=gen(i)).bfloat16().cuda() for i in range(2)]
    want = [E.attend(x, pre, b.cache) for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    ws = [E.alloc_attend_workspace(9, 9, 28, 4, torch.bfloat16) for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            got[i].append(E.attend(q[i], pre, b.cache, ws=ws[i], stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i]) and E.ecokv_device_status(ws[i]) == 0


def test_nothing_to_do():
    b = Batch(1, 2, [1, 1], [4, 5], 8, "bf16")
    empty = torch.zeros(0, 4, D, dtype=torch.bfloat16, device="cuda")
    starts = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert E.attend(empty, None, b.cache, starts).shape == (0, 4, D)
    before = b.dk.clone()
    assert E.append(b.cache, empty[:, :2], empty[:, :2], starts) is None
    assert E.rotate(E.rotary(), torch.zeros(1, 0, dtype=torch.int32, device="cuda"), empty)[0].shape == (0, 4, D)
    assert torch.equal(before.nan_to_num(), b.dk.nan_to_num())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attend_scores_that_jump(dt):
    """A key far above all before it, at each place where a weight's reference can change: within a tile, at its
    end, in the next tile, after masked blocks; and a row whose first keys are far below the rest."""
    g = gen(61)
    T = TYPES[dt]
    n, h_kv = 400, 4
    u = torch.randn(D, generator=g)
    u /= u.norm()
    q = (8 * u + 0.02 * torch.randn(4, h_kv, D, generator=g)).to(T)   # one query head a KV head, four tokens
    b = Batch(23, h_kv, [2, 1, 1], [130, 40, 300], 16, dt)
    heads = []
    for places in ([5, 40, 100], [127, 128, 256], [0], [399, 33]):    # by head
        k = 0.05 * torch.randn(n, D, generator=g)
        for i, at in enumerate(places):
            k[at] += u * (80 + 60 * i)                                # scores 57, 99, 141 units of e apart and more
        heads.append((k.to(T), torch.randn(n, D, generator=g).to(T)))
    heads[2] = (heads[2][0].clone(), heads[2][1])
    heads[2][0][:64] = (-100 * u).to(T)                               # the first keys far below
    pre = E.Prefix(*(torch.stack([h[i] for h in heads]).cuda() for i in range(2)))
    check_attend(b, heads, pre, h_kv, dt, q=q)


@pytest.mark.parametrize("dt,flags", [("f32", 0), ("bf16", E.ECOKV_FLAG_FORCE_SIMT)])
@pytest.mark.parametrize("h,lens,rows", [(8, [700], 0), (32, [1, 129, 4000, 260], 1300), (1, [5000], 20000)])
def test_attend_one_row_an_item_over_many_tiles(h, lens, rows, dt, flags):
    """A head of its own a query head, one token a sequence: a row's maximum and sum pass from tile to tile with no other row between."""
    b = Batch(29, h, [1] * len(lens), lens, 16, dt)
    g = gen(71)
    heads, pre = make_prefix(g, [rows] * h, dt, False)
    q = (2 * torch.randn(len(lens), h, D, generator=g)).to(TYPES[dt])
    check_attend(b, heads, pre if rows else None, h, dt, q=q, flags=flags)


@pytest.mark.parametrize("how", ["stream", "handle", "default"])
def test_helpers_allocate_in_the_order_of_the_stream_they_are_given(how):
    """No workspace and no outputs given, while torch's current stream is busy with readers of memory it has given back."""
    b = Batch(37, 4, [1] * 9, [50 * i + 1 for i in range(9)], 16, "bf16")
    _, pre = make_prefix(gen(3), [900] * 4, "bf16", False)
    q = torch.randn(9, 28, D, generator=gen(1)).bfloat16().cuda()
    r, pos = E.rotary(128, 1e6), torch.arange(9, device="cuda").int()
    want = E.attend(q, pre, b.cache), E.rotate(r, pos, q)[0]
    side = torch.cuda.Stream()
    stream = {"stream": side, "handle": side.cuda_stream, "default": 0}[how]
    busy = side if how == "default" else torch.cuda.current_stream()
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(busy):
            for _ in range(20):
                big @ big
            old = [torch.ones(9, 28, D, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
            kept = [x.clone() for x in old]
            del old
            got = E.attend(q, pre, b.cache, stream=stream), E.rotate(r, pos, q, stream=stream)[0]
            again = E.attend(got[1], pre, b.cache, stream=stream)  # (its workspace may be the one given back)
        (torch.cuda.default_stream() if how == "default" else side).synchronize()
        assert all(torch.equal(x, w) for x, w in zip(got, want))
        assert torch.equal(again, E.attend(want[1], pre, b.cache))
        torch.cuda.synchronize()
        assert all(bool((x == 1).all()) for x in kept)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_rows_that_are_read_may_be_broadcast(dt):
    """One row for every token, or every head: the same as their copies.  An output cannot be one."""
    g, T = gen(81), TYPES[dt]
    r, pos = E.rotary(128, 1e4), torch.arange(40).int().cuda()
    w = (1 + 0.3 * torch.randn(D, generator=g)).to(T).cuda()
    for shape in ((1, 6, D), (40, 1, D), (1, 1, D)):
        x = torch.randn(shape, generator=g).to(T).cuda().expand(40, 6, D)
        want = E.rotate(r, pos, x.contiguous(), q_norm=w)[0]
        assert torch.equal(E.rotate(r, pos, x, q_norm=w)[0], want)
        b = [Batch(83, 6, [40], [50], 16, dt) for _ in range(2)]
        for c, k in zip(b, (x, x.contiguous())):
            E.append(c.cache, k, k, c.starts.cuda(), r, pos)
        assert torch.equal(b[0].dk.nan_to_num(), b[1].dk.nan_to_num())
        assert torch.equal(b[0].dv.nan_to_num(), b[1].dv.nan_to_num())
        with pytest.raises(E.EcokvError) as e:
            E.rotate(r, pos, want, q_out=x)
        assert e.value.code == E.ECOKV_ERR_INVALID_ARG


def jump_rows(dt, low, at=(40, 77, 149), own=(1.0, 1.0, 1.0), heads=33):
    """One KV head, a query head a row, scores exact in any order of sums: `low` for the first 40 keys, then three of
    a row's own (`own` / 16 times -16 .. 16), in units of log2 at the scale returned with them."""
    scale = float(torch.tensor(0.0625 / math.log2(math.e), dtype=torch.float32))
    assert float(torch.tensor(math.log2(math.e) * scale, dtype=torch.float32)) == 0.0625
    T, n = TYPES[dt], 150
    q = torch.zeros(1, heads, D)
    q[0, :, 0] = torch.arange(heads) - heads // 2
    q[0, :, 1] = 32
    k = torch.zeros(n, D)
    k[:, 1] = low / 2            # 32 x low / 2 / 16
    k[list(at), 0] = torch.tensor(own)
    k[list(at), 1] = 0
    return q.to(T), k.to(T), scale


@pytest.mark.parametrize("dt,flags", [("bf16", 0), ("bf16", E.ECOKV_FLAG_FORCE_SIMT), ("f32", 0)])
@pytest.mark.parametrize("low", [-63, -60, -15, -3])
def test_attend_log_sum_near_zero(low, dt, flags):
    """Sums near one whose first keys lie far below: the logarithm is rounded as a number of its own size, not of the
    first keys'.  An exponential is off by 2^-22, a sum of the few weights that count by 3 u and the lower ones'
    share, the logarithm of a mantissa by 2 u, the result (2 at most, times ln 2) by 4 u more."""
    # (in one tile of keys: the largest of another's would be the reference)
    q, k, scale = jump_rows(dt, low, (40, 77, 120), (1.0, 2.0, -1.0))
    v = torch.randn(k.shape, generator=gen(91)).to(TYPES[dt])
    pre = E.Prefix(k[None].cuda(), v[None].cuda())
    lse = torch.zeros(1, q.shape[1], device="cuda")
    E.attend(q.cuda(), pre, None, scale=scale, lse=lse, flags=flags)
    want = torch.logsumexp(q[0].double() @ k.double().t() * scale, -1)
    err = (lse[0].cpu().double() - want).abs()
    assert bool((err <= 2.0 ** -22 + 9 * U + 150 * U * 2.0 ** (low + 1)).all()), float(err.max())


@pytest.mark.parametrize("dt,flags", [("bf16", 0), ("bf16", E.ECOKV_FLAG_FORCE_SIMT), ("f32", 0)])
@pytest.mark.parametrize("low", [-63, -40, -17, -16, -15.5, -8])
def test_attend_large_values_after_a_jump(low, dt, flags):
    """Values near the bound of the header where the scores rise: the unnormalised sums stay finite."""
    q, k, scale = jump_rows(dt, low)
    v = (torch.randn(k.shape, generator=gen(92)).clamp(-4, 4) * 2.0 ** 83).to(TYPES[dt])
    b = Batch(93, 1, [1], [0], 16, dt)
    check_attend(b, [(k, v)], E.Prefix(k[None].cuda(), v[None].cuda()), q.shape[1], dt, q=q, flags=flags, scale=scale)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attend_room_of_the_table_does_not_count(dt):
    """A table with room for 2^21 slots a sequence and many tokens: the same bits as with a table of the slots in use."""
    g, page, n = gen(97), 4096, 4500
    k, v = torch.randn(2, 4, 1, page, D, generator=g).to(TYPES[dt]).cuda()
    q = torch.randn(n, 64, D, generator=g).to(TYPES[dt]).cuda()
    lengths, starts = torch.tensor([5000, 10]).int().cuda(), torch.tensor([0, n - 10, n]).int().cuda()
    out = []
    for cols in (2, 512):
        table = torch.full((2, cols), 2 ** 30, dtype=torch.int32)
        table[0, :2], table[1, 0] = torch.tensor([2, 1]), 3
        out.append(E.attend(q, None, E.PagedCache(k, v, table.cuda(), lengths), starts))
    assert torch.equal(out[0], out[1]) and bool(out[0].float().abs().max() > 0.1)


def test_attend_starts_that_overlap_past_32_bits():
    """Starts that go up and down, so that each of many sequences holds all tokens: said in the status, no slot is read."""
    # (16 of 32 sequences of 16384 tokens over 2^22 slots: 2^32 units of work and more, were they walked)
    n, page, cols, batch = 16384, 4096, 1024, 32
    k, v = torch.randn(2, 1, 1, page, D, generator=gen(98)).bfloat16().cuda()
    q = torch.randn(n, 64, D, generator=gen(99)).bfloat16().cuda()
    starts = torch.tensor([0, n] * (batch // 2) + [0]).int().cuda()
    cache = E.PagedCache(k, v, torch.zeros(batch, cols, dtype=torch.int32, device="cuda"),
                         torch.full((batch,), cols * page, dtype=torch.int32, device="cuda"))
    ws = E.alloc_attend_workspace(n, batch, 64, 1, torch.bfloat16)
    lse = torch.zeros(n, 64, device="cuda")
    out = E.attend(q, None, cache, starts, ws=ws, lse=lse)
    assert E.ecokv_device_status(ws) == E.ECOKV_ERR_DEVICE_INDEX
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
